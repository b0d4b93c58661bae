// C ABI of the norm and the gated feed-forward block (declared in
// include/moe.h): host-side argument validation, workspace carving and the
// launch sequences.  Every check runs before the first launch; nothing here
// allocates, synchronises or keeps state.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "../../include/moe.h"
#include "dense.hpp"

namespace {

constexpr size_t kAlign = 256;
static_assert(MOE_MAX_WIDTH == moe::kMostWidth, "the widths that kernels are made for");

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

template <class... P>
bool aligned16(const P*... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & 15u) == 0;
}

// An array's bytes; none of them where it is NULL or not used.
struct Span {
  uintptr_t p;
  size_t n;
  Span(const void* at, size_t bytes) : p(reinterpret_cast<uintptr_t>(at)), n(at ? bytes : 0) {}
};
// Whether `out` meets none of the others, but for those in `same` that start where it does.
bool apart(Span out, std::initializer_list<Span> others, std::initializer_list<Span> same = {}) {
  auto meet = [&](const Span& o) { return o.n && out.n && out.p < o.p + o.n && o.p < out.p + out.n; };
  for (const Span& o : others)
    if (meet(o)) return false;
  for (const Span& o : same)
    if (o.p != out.p && meet(o)) return false;
  return true;
}

bool norm_sizes(int T, int H) { return T >= 0 && T <= MOE_MAX_ROWS && H >= 1 && H <= MOE_MAX_WIDTH; }

moe_status check_norm(int T, int H, int kind, int dtype) {
  if (!norm_sizes(T, H)) return MOE_ERR_SHAPE;
  if (kind != MOE_NORM_LAYER && kind != MOE_NORM_RMS) return MOE_ERR_UNSUPPORTED;
  if (dtype != MOE_DT_F32 && dtype != MOE_DT_BF16 && dtype != MOE_DT_F16) return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

size_t bytes_of(int dtype) { return dtype == MOE_DT_F32 ? 4 : 2; }

bool ffn_sizes(const moe_ffn_args* a) {
  return a->T >= 0 && a->T <= MOE_MAX_ROWS && a->H >= 8 && a->H <= MOE_MAX_WIDTH && a->H % 8 == 0 && a->I >= 8 &&
         a->I <= MOE_MAX_WIDTH && a->I % 8 == 0;
}

moe_status check_ffn(const moe_ffn_args* a) {
  if (!a) return MOE_ERR_NULL;
  if (!ffn_sizes(a)) return MOE_ERR_SHAPE;
  if (a->dtype != MOE_DT_BF16 && a->dtype != MOE_DT_F16) return MOE_ERR_UNSUPPORTED;
  if (a->act != MOE_ACT_SILU && a->act != MOE_ACT_GELU_TANH) return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

// The arrays of a block's call.
struct FfnSpans {
  Span x, w1, w2, pre, ws;
  FfnSpans(const moe_ffn_args* a, const void* at, size_t ws_bytes)
      : x(a->x, rows(a) * a->H * 2), w1(a->w1, size_t{4} * a->I * a->H), w2(a->w2, size_t{2} * a->I * a->H),
        pre(a->pre, rows(a) * a->I * 8), ws(at, ws_bytes) {}
  static size_t rows(const moe_ffn_args* a) { return static_cast<size_t>(a->T); }
};

// Workspace: forward h, then the partial products of a split K; backward dpre, h,
// then those.  Offsets from the start.
struct FfnLayout {
  size_t dpre, h, part, total;
};
FfnLayout forward_layout(const moe_ffn_args* a) {
  FfnLayout L{};
  L.part = align_up(static_cast<size_t>(a->T) * a->I * 2);
  L.total = L.part + align_up(std::max(moe::dense_gemm_workspace_bytes(moe::kRowRow, moe::kGlu, a->T, a->I, a->H),
                                       moe::dense_gemm_workspace_bytes(moe::kRowRow, moe::kStore, a->T, a->H, a->I)));
  return L;
}
FfnLayout backward_layout(const moe_ffn_args* a) {
  FfnLayout L{};
  L.h = align_up(static_cast<size_t>(a->T) * 2 * a->I * 2);
  L.part = L.h + align_up(static_cast<size_t>(a->T) * a->I * 2);
  L.total = L.part + align_up(std::max({moe::dense_gemm_workspace_bytes(moe::kRowCol, moe::kDglu, a->T, a->I, a->H),
                                        moe::dense_gemm_workspace_bytes(moe::kRowCol, moe::kStore, a->T, a->H, 2 * a->I),
                                        moe::dense_gemm_workspace_bytes(moe::kColCol, moe::kStore, 2 * a->I, a->H, a->T),
                                        moe::dense_gemm_workspace_bytes(moe::kColCol, moe::kStore, a->H, a->I, a->T)}));
  return L;
}

template <class T>
T* at(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

}  // namespace

extern "C" {

moe_status moe_norm_forward(const void* x, const void* residual, const void* weight, const void* bias, int T, int H,
                            int kind, int dtype, float eps, void* y, void* sum, float* mean, float* rstd,
                            hipStream_t stream) {
  const moe_status st = check_norm(T, H, kind, dtype);
  if (st != MOE_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps) || (kind == MOE_NORM_RMS && bias)) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!x || !weight || !y || (residual && !sum)) return MOE_ERR_NULL;
  if (!aligned16(x, residual, weight, bias, y, sum) || !aligned16(mean, rstd)) return MOE_ERR_ALIGN;
  const size_t n = static_cast<size_t>(T) * H * bytes_of(dtype), row = H * bytes_of(dtype), stat = static_cast<size_t>(T) * 4;
  const Span sx{x, n}, sr{residual, n}, sw{weight, row}, sb{bias, row}, sy{y, n}, ss{residual ? sum : nullptr, n},
      sm{kind == MOE_NORM_LAYER ? mean : nullptr, stat}, srs{rstd, stat};
  if (!apart(sy, {sw, sb, ss, sm, srs}, {sx, sr}) || !apart(ss, {sw, sb, sm, srs}, {sx, sr}) ||
      !apart(sm, {sx, sr, sw, sb, srs}) || !apart(srs, {sx, sr, sw, sb}))
    return MOE_ERR_UNSUPPORTED;
  const moe::NormForward a{x, residual, weight, bias, T, H, eps, y, sum, mean, rstd};
  return moe::launch_norm_forward(dtype, kind, a, stream) == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

size_t moe_norm_backward_workspace_bytes(int T, int H) {
  return norm_sizes(T, H) ? align_up(moe::norm_backward_workspace_bytes(T, H)) : 0;
}

moe_status moe_norm_backward(const void* dy, const void* x, const void* weight, const float* mean, const float* rstd,
                             const void* dsum, int T, int H, int kind, int dtype, void* dx, float* dweight,
                             float* dbias, void* ws, size_t ws_bytes, hipStream_t stream) {
  const moe_status st = check_norm(T, H, kind, dtype);
  if (st != MOE_OK) return st;
  if (kind == MOE_NORM_RMS && dbias) return MOE_ERR_UNSUPPORTED;
  if (T > 0 && (!dy || !x || !weight || !rstd || !dx || (kind == MOE_NORM_LAYER && !mean))) return MOE_ERR_NULL;
  if (!aligned16(dy, x, weight, dsum, dx, ws) || !aligned16(mean, rstd, dweight, dbias)) return MOE_ERR_ALIGN;
  const bool sums = dweight || dbias;
  if (T == 0 && !sums) return MOE_OK;
  const size_t need = sums ? align_up(moe::norm_backward_workspace_bytes(T, H)) : 0;
  if (need && (!ws || ws_bytes < need)) return MOE_ERR_WORKSPACE;
  const size_t n = static_cast<size_t>(T) * H * bytes_of(dtype), row = H * bytes_of(dtype), stat = static_cast<size_t>(T) * 4,
               column = static_cast<size_t>(H) * 4;
  const Span sdy{dy, n}, sx{x, n}, sw{weight, row}, sm{kind == MOE_NORM_LAYER ? mean : nullptr, stat}, srs{rstd, stat},
      sds{dsum, n}, sdw{dweight, column}, sdb{dbias, column}, sws{ws, need};
  if (!apart({dx, n}, {sx, sw, sm, srs, sdw, sdb, sws}, {sdy, sds}) || !apart(sdw, {sdy, sx, sw, sm, srs, sds, sdb, sws}) ||
      !apart(sdb, {sdy, sx, sw, sm, srs, sds, sws}) || !apart(sws, {sdy, sx, sw, sm, srs, sds}))
    return MOE_ERR_UNSUPPORTED;
  const moe::NormBackward a{dy, x, weight, dsum, mean, rstd, T, H, dx, dweight, dbias, sums ? static_cast<float*>(ws) : nullptr};
  return moe::launch_norm_backward(dtype, kind, a, stream) == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

size_t moe_ffn_workspace_bytes(const moe_ffn_args* a) { return a && ffn_sizes(a) ? forward_layout(a).total : 0; }

size_t moe_ffn_backward_workspace_bytes(const moe_ffn_args* a) {
  return a && ffn_sizes(a) ? backward_layout(a).total : 0;
}

moe_status moe_ffn_forward(const moe_ffn_args* a, void* ws, size_t ws_bytes, hipStream_t stream) {
  const moe_status st = check_ffn(a);
  if (st != MOE_OK) return st;
  if (a->T == 0) return MOE_OK;
  if (!a->x || !a->w1 || !a->w2 || !a->y) return MOE_ERR_NULL;
  if (!aligned16(a->x, a->w1, a->w2, a->add, a->y) || !aligned16(a->pre)) return MOE_ERR_ALIGN;
  const FfnLayout L = forward_layout(a);
  if (!ws || ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  if (!aligned16(ws)) return MOE_ERR_ALIGN;
  const FfnSpans sp(a, ws, L.total);
  const Span add{a->add, sp.x.n};
  if (!apart({a->y, sp.x.n}, {sp.w1, sp.w2, sp.pre, sp.ws}, {sp.x, add}) || !apart(sp.pre, {sp.x, sp.w1, sp.w2, add, sp.ws}) ||
      !apart(sp.ws, {sp.x, sp.w1, sp.w2, add}))
    return MOE_ERR_UNSUPPORTED;

  moe::DenseGemm g{};
  g.act = a->act;
  g.part = at<float>(ws, L.part);
  g.a = a->x;
  g.b = a->w1;
  g.M = a->T;
  g.N = a->I;
  g.K = a->H;
  g.c = at<void>(ws, L.h);
  g.pre = a->pre;
  if (moe::launch_dense_gemm(a->dtype, moe::kRowRow, moe::kGlu, g, stream) != hipSuccess) return MOE_ERR_HIP;
  g.a = g.c;
  g.b = a->w2;
  g.N = a->H;
  g.K = a->I;
  g.c = a->y;
  g.add = a->add;
  if (moe::launch_dense_gemm(a->dtype, moe::kRowRow, moe::kStore, g, stream) != hipSuccess) return MOE_ERR_HIP;
  return MOE_OK;
}

moe_status moe_ffn_backward(const moe_ffn_args* a, void* ws, size_t ws_bytes, hipStream_t stream) {
  const moe_status st = check_ffn(a);
  if (st != MOE_OK) return st;
  if (!a->dx && !a->dw1 && !a->dw2) return MOE_OK;
  if (a->T > 0 && (!a->dy || !a->w2 || !a->pre || (a->dx && !a->w1) || (a->dw1 && !a->x))) return MOE_ERR_NULL;
  if (!aligned16(a->x, a->w1, a->w2, a->dy, a->dx, a->dw1, a->dw2) || !aligned16(a->pre)) return MOE_ERR_ALIGN;
  const FfnLayout L = backward_layout(a);
  if (L.total && (!ws || ws_bytes < L.total)) return MOE_ERR_WORKSPACE;
  if (!aligned16(ws)) return MOE_ERR_ALIGN;
  const FfnSpans sp(a, ws, L.total);
  const size_t n = static_cast<size_t>(a->T) * a->H * 2;
  const Span dy{a->dy, n}, x{a->dw1 ? a->x : nullptr, n}, w1{a->dx ? a->w1 : nullptr, sp.w1.n}, dx{a->dx, n},
      dw1{a->dw1, sp.w1.n}, dw2{a->dw2, sp.w2.n};
  if (!apart(dx, {dy, x, w1, sp.w2, sp.pre, dw1, dw2, sp.ws}) || !apart(dw1, {dy, x, w1, sp.w2, sp.pre, dw2, sp.ws}) ||
      !apart(dw2, {dy, x, w1, sp.w2, sp.pre, sp.ws}) || !apart(sp.ws, {dy, x, w1, sp.w2, sp.pre}))
    return MOE_ERR_UNSUPPORTED;

  moe::DenseGemm g{};
  g.act = a->act;
  g.part = at<float>(ws, L.part);
  void* const dpre = at<void>(ws, L.dpre);
  void* const h = at<void>(ws, L.h);
  if (a->T > 0) {
    g.a = a->dy;
    g.b = a->w2;
    g.M = a->T;
    g.N = a->I;
    g.K = a->H;
    g.c = dpre;
    g.pre_in = a->pre;
    g.h = a->dw2 ? h : nullptr;
    if (moe::launch_dense_gemm(a->dtype, moe::kRowCol, moe::kDglu, g, stream) != hipSuccess) return MOE_ERR_HIP;
  }
  auto product = [&](int layout, const void* pa, const void* pb, int M, int N, int K, void* c) {
    g.a = pa;
    g.b = pb;
    g.M = M;
    g.N = N;
    g.K = K;
    g.c = c;
    return M == 0 || moe::launch_dense_gemm(a->dtype, layout, moe::kStore, g, stream) == hipSuccess;
  };
  if (a->dx && !product(moe::kRowCol, dpre, a->w1, a->T, a->H, 2 * a->I, a->dx)) return MOE_ERR_HIP;
  if (a->dw1 && !product(moe::kColCol, dpre, a->x, 2 * a->I, a->H, a->T, a->dw1)) return MOE_ERR_HIP;
  if (a->dw2 && !product(moe::kColCol, a->dy, h, a->H, a->I, a->T, a->dw2)) return MOE_ERR_HIP;
  return MOE_OK;
}

}  // extern "C"
