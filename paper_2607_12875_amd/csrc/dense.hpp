// Internal launchers of the dense operators (host side): the norm and the gated
// feed-forward block.  Shapes are validated by the C ABI layer (dense_api.hip)
// before any of these is called.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

namespace moe {

// Element types and kinds, the values of moe_dtype, moe_norm_kind, moe_act.
constexpr int kF32 = 0, kBf16 = 1, kF16 = 2;
constexpr int kLayerNorm = 0, kRmsNorm = 1;
constexpr int kSilu = 0, kGeluTanh = 1;
constexpr int kMostWidth = 65536;  // MOE_MAX_WIDTH

struct NormForward {
  const void *x, *residual, *weight, *bias;  // residual, bias: or null
  int T, H;
  float eps;
  void *y, *sum;       // sum: with a residual
  float *mean, *rstd;  // or null
};
struct NormBackward {
  const void *dy, *x, *weight, *dsum;  // dsum: or null
  const float *mean, *rstd;            // mean: layer only
  int T, H;
  void* dx;
  float *dweight, *dbias;  // each or null
  float* part;             // partial column sums, norm_backward_workspace_bytes
};
size_t norm_backward_workspace_bytes(int T, int H);
hipError_t launch_norm_forward(int dtype, int kind, const NormForward& a, hipStream_t s);
hipError_t launch_norm_backward(int dtype, int kind, const NormBackward& a, hipStream_t s);

// C[m][n] = sum_k A(m,k) B(n,k) over 16-bit operands.  A row operand holds
// element (r, k) at r * ld + k, a column operand at k * ld + r.
enum DenseEpilogue {
  kStore,  // c = C (+ add)
  kGlu,    // B is [2N, K], gate rows then up rows: h = act(gate) * up, and pre
  kDglu,   // C = dh: dpre = [dh * up * act'(gate), dh * act(gate)], and h again
};
struct DenseGemm {
  const void *a, *b;
  int M, N, K;       // kGlu: N columns of h
  int act;
  void* c;           // [M, N]
  const void* add;   // kStore: [M, N] or null
  const float* pre_in;  // kDglu: [M, 2N]
  float* pre;        // kGlu: [M, 2N] or null
  void* h;           // kDglu: [M, N] or null; c is dpre [M, 2N] there
  float* part;       // fp32 partial products where K is split
};
// Operand layouts of the products that the block needs.
enum DenseLayout { kRowRow, kRowCol, kColCol };
// Bytes of part; never fewer for more rows of the block (M, K where both operands are columns).
size_t dense_gemm_workspace_bytes(int layout, int epi, int M, int N, int K);
hipError_t launch_dense_gemm(int dtype, int layout, int epi, const DenseGemm& g, hipStream_t s);

// The forward products for few rows of A, where that is the faster form.
bool dense_rows_fits(int layout, int epi, int M, int N, int K);
hipError_t launch_dense_rows(int dtype, int epi, const DenseGemm& g, hipStream_t s);

}  // namespace moe
