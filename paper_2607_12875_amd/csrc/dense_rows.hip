// The feed-forward block's forward products for few rows (decode): C[m][n] =
// sum_k A(m,k) B(n,k) with up to 32 rows of A.  Every weight byte is read once, and
// that is most of the time there is.  A workgroup owns sixteen rows of B (kGlu: eight
// gate and eight up, of the same columns) and its four waves share K out in pieces
// of 256 elements.  HBM wants long runs: a load instruction takes 512 contiguous
// bytes of each of two rows, which the wave turns over in LDS of its own into the
// fragments of v_mfma_f32_16x16x32 (loading those straight from memory, 64 bytes of
// sixteen rows at a time, took 78 us for 16 tokens, 4096 x 11264; 56 this way, 61 where
// every call has other weights).  The next piece is in flight meanwhile.  The waves'
// sums meet in LDS, in wave order.  Eight waves per workgroup (69 us, the same weights)
// and 32 rows of B (61 us) keep fewer pieces in flight.  One token, 4096 x 11264: 34
// us for the first product's 184 MB, 18 for the second's 92, each with about 3 us of
// launch and first loads.  Every workgroup reads all of A from L2: at 16 tokens, 4096
// wide, as many bytes as its weights (37 + 20 us).
#include <algorithm>

#include "common.hpp"
#include "dense.hpp"
#include "dense_finish.hpp"
#include "dense_math.hpp"

namespace moe {

namespace {

typedef __amdgpu_buffer_rsrc_t Buffer;

__device__ __forceinline__ u32x4 load16(Buffer b, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0));
}

constexpr uint32_t kPast = 0x40000000u;  // an offset behind every buffer, alone and twice: reads zero

// LDS slot of 16-byte chunk c of a row of 32: sixteen rows' chunks of one fragment lie in different banks.
__device__ __forceinline__ int slot(int row, int c) { return row * 32 + (c ^ (row & 15)); }

template <class E, int MT, int EPI>
__global__ __launch_bounds__(256) void dense_rows_kernel(DenseGemm g) {
  constexpr bool DUAL = EPI == kGlu;
  constexpr int NW = 4, BR = 16, NC = DUAL ? BR / 2 : BR, PIECE = 256;
  constexpr int PITCH = BR + 4;
  constexpr int TR = MT * 16;  // rows turned over at once
  constexpr int kTurn = NW * TR * PIECE * 2, kRed = NW * MT * 16 * PITCH * 4;
  __shared__ __attribute__((aligned(16))) uint8_t smem[kTurn > kRed ? kTurn : kRed];
  const int lane = lane_id(), wave = threadIdx.x / kWave, l16 = lane & 15, kg = lane >> 4, lr = lane >> 5, lc = lane & 31;
  const int n0 = blockIdx.x * NC;

  // Buffers: A's rows; B's rows of this workgroup (gate and up apart).  A row
  // that is not there lies past the end and reads as zeros.
  const uint16_t* const pb = static_cast<const uint16_t*>(g.b) + static_cast<size_t>(n0) * g.K;
  const int rows = min(NC, g.N - n0);
  const uint32_t ld = static_cast<uint32_t>(g.K) * 2u;
  const Buffer ba = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(g.a), 0, g.M * ld, 0x00020000);
  const Buffer b0 = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(pb), 0, rows * ld, 0x00020000);
  const Buffer b1 = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(pb + (DUAL ? static_cast<size_t>(g.N) * g.K : 0)),
                                                      0, rows * ld, 0x00020000);

  // one piece of the rows: 16 bytes per lane of two rows per load
  auto load_b = [&](u32x4 (&x)[8], int k0) {
    const uint32_t at = k0 + lc * 8 < g.K ? k0 * 2u + lc * 16u : kPast;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int half = DUAL && i >= 4, r = (half ? i - 4 : i) * 2 + lr;
      x[i] = load16(half ? b1 : b0, (r < rows ? r * ld : kPast) + at);
    }
  };
  u32x4 xa[8 * MT];
  auto load_a = [&](int k0) {
    const uint32_t at = k0 + lc * 8 < g.K ? k0 * 2u + lc * 16u : kPast;
#pragma unroll
    for (int i = 0; i < 8 * MT; ++i) {
      const int r = i * 2 + lr;
      if (i * 2 < g.M) xa[i] = load16(ba, (r < g.M ? r * ld : kPast) + at);  // uniform: pairs of rows that are there
    }
  };
  f32x4 acc[MT] = {};
  u32x4* const turn = reinterpret_cast<u32x4*>(smem) + wave * TR * 32;
  // the wave's own LDS: other lanes' writes come before the reads that follow, and the reverse
  auto turned = [] {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_wave_barrier();
  };
  auto multiply = [&](const u32x4 (&xb)[8]) {
    u32x4 fa[8][MT];
#pragma unroll
    for (int i = 0; i < 8 * MT; ++i)
      if (i * 2 < g.M) turn[slot(i * 2 + lr, lc)] = xa[i];
    turned();
#pragma unroll
    for (int h = 0; h < 8; ++h)
#pragma unroll
      for (int m = 0; m < MT; ++m) fa[h][m] = turn[slot(m * 16 + l16, h * 4 + kg)];
    turned();
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[slot(i * 2 + lr, lc)] = xb[i];
    turned();
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      const u32x4 fb = turn[slot(l16, h * 4 + kg)];
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m] = mfma16<E>(fb, fa[h][m], acc[m]);
    }
    turned();
  };
  // A's piece (from L2) goes out ahead of B's next one, so that it is not waited for behind it
  u32x4 x[8], y[8];
  const int step = NW * PIECE;
  int k0 = wave * PIECE;
  if (k0 < g.K) load_b(x, k0);
  while (k0 < g.K) {  // uniform in the wave
    load_a(k0);
    if (k0 + step < g.K) load_b(y, k0 + step);
    multiply(x);
    k0 += step;
    if (k0 >= g.K) break;
    load_a(k0);
    if (k0 + step < g.K) load_b(x, k0 + step);
    multiply(y);
    k0 += step;
  }
  __syncthreads();
  auto red = reinterpret_cast<float(*)[MT * 16][PITCH]>(smem);

  // lane: row l16 of A, four B rows from 4 kg on
#pragma unroll
  for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4*>(&red[wave][m * 16 + l16][kg * 4]) = acc[m];
  __syncthreads();
  const int count = min(g.M, MT * 16) * BR;
  for (int e = threadIdx.x; e < count; e += NW * 64) {
    float v = red[0][e / BR][e % BR];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += red[w][e / BR][e % BR];
    red[0][e / BR][e % BR] = v;
  }
  __syncthreads();
  constexpr int GROUPS = NC / 8;  // of eight columns
  for (int e = threadIdx.x; e < g.M * GROUPS; e += NW * 64) {
    const int m = e / GROUPS, c = e % GROUPS * 8, n = n0 + c;
    if (n >= g.N) continue;
    Beside<E, EPI> x;
    x.load(g, m, n);
    finish8<E, EPI>(g, m, n, load8<float>(&red[0][m][c]), DUAL ? load8<float>(&red[0][m][NC + c]) : f32x8{}, x);
  }
}

template <class E, int EPI>
hipError_t rows(const DenseGemm& g, hipStream_t s) {
  constexpr int NC = EPI == kGlu ? 8 : 16;
  const unsigned grid = (g.N + NC - 1) / NC;
  if (g.M <= 16) dense_rows_kernel<E, 1, EPI><<<grid, 256, 0, s>>>(g);
  else dense_rows_kernel<E, 2, EPI><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace

// Up to 16 rows always.  A second fragment of rows takes the registers that keep
// the weights coming, which costs large weights more than the tile kernels' split of
// K and their joining launch: 17 rows, 4096 x 1408, 14.4 us here and 17.7 there, 24
// rows, 2048 x 1408, 11.7 and 15.7, 32 rows, 5120 x 1536, 22.4 and 20.4, 7168 x 2048,
// 30.2 and 25.5.
bool dense_rows_fits(int layout, int epi, int M, int N, int K) {
  if (layout != kRowRow || epi == kDglu || M > 32) return false;
  return M <= 16 || static_cast<long>(N) * K * (epi == kGlu ? 2 : 1) <= 3L << 22;
}

hipError_t launch_dense_rows(int dtype, int epi, const DenseGemm& g, hipStream_t s) {
  if (dtype == kBf16) return epi == kGlu ? rows<bf16_t, kGlu>(g, s) : rows<bf16_t, kStore>(g, s);
  return epi == kGlu ? rows<f16_t, kGlu>(g, s) : rows<f16_t, kStore>(g, s);
}

}  // namespace moe
