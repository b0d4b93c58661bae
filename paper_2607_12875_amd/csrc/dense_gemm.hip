// The products of the gated feed-forward block (a shared expert beside the
// routed ones, or a dense layer), 16-bit operands and fp32 sums on
// v_mfma_f32_32x32x16:
//   forward   pre = x W1^T -> h = act(gate) * up in the epilogue;  y = h W2^T (+ add)
//   backward  dh = dy W2 -> dpre = [dh u act'(g), dh act(g)] and h in the epilogue;
//             dx = dpre W1;  dW1 = dpre^T x;  dW2 = dy^T h
// One tile kernel serves the six: an operand lies in memory with its reduction
// index innermost (a row operand) or outermost (a column operand), and goes to
// LDS as it lies.  A fragment of a row operand is one ds_read_b128; of a column
// operand two ds_read_b64_tr_b16, which transpose 4 x 16 blocks on the way.
#include <algorithm>

#include "common.hpp"
#include "dense.hpp"
#include "dense_math.hpp"
#include "lds_dma.hpp"

namespace moe {

constexpr int kBK = 64;  // K elements per step: 128 bytes, one line of a row operand

// Sixteen bytes per lane from a bounds-checked buffer to LDS: lane l reads
// offset voff and lands at `lds` + 16 l.  Lanes past the buffer's end write zeros.
__device__ __forceinline__ void bdma16(const u32x4& rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}
__device__ __forceinline__ u32x4 buffer_of(uint64_t base, uint32_t bytes) {
  u32x4 r;
  r.x = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base));
  r.y = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base >> 32) & 0xFFFFu);
  r.z = __builtin_amdgcn_readfirstlane(bytes);
  r.w = 0x00020000u;
  return r;
}

// One operand's tile of R rows (COL: columns) by kBK: its copies and fragments.
// Row operand: 128-byte LDS rows of eight chunks, row r's chunk c in slot
// c ^ ((r >> 1) & 7).  Column operand: LDS row k holds the R elements of index
// k, its chunk c in slot c ^ tswz(k): the four rows that one transposing read
// takes lie in different banks.
template <int R, bool COL, int NW, int PARTS>
struct Operand {
  static constexpr int kBytes = R * kBK * 2;
  static constexpr int kCopies = kBytes / 1024 / NW;  // per wave and step
  static_assert(kCopies >= 1 && kCopies * NW * 1024 == kBytes && (kCopies % PARTS == 0), "copies");
  static constexpr int kChunks = COL ? R / 8 : 8;  // per LDS row
  static constexpr int kRows = 64 / kChunks;       // LDS rows per copy
  static_assert(!COL || (R >= 64 && PARTS == 1), "column tiles");
  __device__ static int tswz(int k) { return R == 64 ? (k & 2) << 1 : (k & 3) << 2; }

  uint64_t base[PARTS];
  uint32_t left[PARTS];  // row: bytes from the base to the end of the tile's rows
  uint32_t voff[kCopies];
  int ld;

  // row operand: `at` the first of `rows` rows that exist from the tile's start
  __device__ void rows(int part, const void* at, int rows, int ld_, int k0) {
    ld = ld_;
    base[part] = reinterpret_cast<uint64_t>(at) + static_cast<uint64_t>(k0) * 2;
    left[part] = static_cast<uint32_t>(max(0, min(rows, R / PARTS))) * static_cast<uint32_t>(ld_) * 2u;
    left[part] = left[part] ? left[part] - k0 * 2u : 0u;
  }
  // column operand: column m0 of the rows from k0 on
  __device__ void cols(const void* at, int m0, int ld_, int k0) {
    ld = ld_;
    base[0] = reinterpret_cast<uint64_t>(at) + (static_cast<uint64_t>(k0) * ld_ + m0) * 2;
    left[0] = m0 * 2u;
  }
  __device__ void offsets(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = ((i % (kCopies / PARTS)) * NW + wave) * kRows + lane / kChunks;  // row within its part
      const int c = (lane % kChunks) ^ (COL ? tswz(r) : (r >> 1) & 7);
      voff[i] = static_cast<uint32_t>(r) * static_cast<uint32_t>(ld) * 2u + c * 16u;
    }
  }
  // The copies of the step that starts at k (of K), into LDS at `lds`; then
  // the operand stands at the next step.
  __device__ void issue(int k, int K, int wave, int lane, uint32_t lds) {
    if constexpr (!COL) {
      if (k + kBK > K) {  // uniform: the last step of a ragged K; chunks past K copy zeros
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int r = ((i % (kCopies / PARTS)) * NW + wave) * kRows + lane / kChunks;
          const int c = (lane % kChunks) ^ ((r >> 1) & 7);
          if (k + c * 8 >= K) voff[i] = 0x80000000u;
        }
      }
    }
    u32x4 d[PARTS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
      d[p] = buffer_of(base[p], COL ? static_cast<uint32_t>(min(K - k, kBK)) * static_cast<uint32_t>(ld) * 2u - left[p] : left[p]);
#pragma unroll
    for (int i = 0; i < kCopies; ++i) bdma16(d[i / (kCopies / PARTS)], voff[i], lds + (i * NW + wave) * 1024);
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      base[p] += COL ? static_cast<uint64_t>(ld) * kBK * 2 : kBK * 2;
      if (!COL) left[p] = left[p] > kBK * 2u ? left[p] - kBK * 2u : 0u;
    }
  }
  // Fragment of the 32 rows (columns) from r0 on at K substep kk: eight
  // consecutive k of group lane / 32 for row lane % 32.
  __device__ static u32x4 frag(uint32_t lds, int r0, int kk, int lane) {
    if constexpr (!COL) {
      const int r = r0 + (lane & 31);
      return lds16(lds + r * 128 + (((2 * kk + (lane >> 5)) ^ ((r >> 1) & 7)) << 4));
    } else {
      // lane group of 16: columns 16 ((lane >> 4) & 1) .. of the block, rows 8 (lane >> 5) ..
      const int k = (lane & 15) >> 2;  // and k + 4
      const int c = r0 / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
      const uint32_t at = lds + (16 * kk + 8 * (lane >> 5) + k) * (R * 2) + ((c ^ tswz(k)) << 4) + ((lane & 1) << 3);
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* lp;
      const i32x2 lo = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)at));
      const i32x2 hi = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(at + 4 * R * 2)));
      return u32x4{static_cast<uint32_t>(lo.x), static_cast<uint32_t>(lo.y), static_cast<uint32_t>(hi.x),
                   static_cast<uint32_t>(hi.y)};
    }
  }
};

// The epilogue on four columns of one row; SPLIT products come from the partial sums.
template <class E, int EPI>
__device__ __forceinline__ void finish4(const DenseGemm& g, int m, int n, const f32x4& c, const f32x4& up) {
  const size_t at = static_cast<size_t>(m) * g.N + n;
  const size_t at2 = static_cast<size_t>(m) * 2 * g.N + n;
  if constexpr (EPI == kStore) {
    f32x4 v = c;
    if (g.add) v += load4<E>(static_cast<const E*>(g.add) + at);
    store4<E>(static_cast<E*>(g.c) + at, v);
  } else if constexpr (EPI == kGlu) {
    if (g.pre) {
      *reinterpret_cast<f32x4*>(g.pre + at2) = c;
      *reinterpret_cast<f32x4*>(g.pre + at2 + g.N) = up;
    }
    f32x4 h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = act_of(g.act, c[i]) * up[i];
    store4<E>(static_cast<E*>(g.c) + at, h);
  } else {
    const f32x4 gt = *reinterpret_cast<const f32x4*>(g.pre_in + at2);
    const f32x4 u = *reinterpret_cast<const f32x4*>(g.pre_in + at2 + g.N);
    f32x4 dg, du, h;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, da;
      act_and_slope(g.act, gt[i], a, da);
      dg[i] = c[i] * u[i] * da;
      du[i] = c[i] * a;
      h[i] = a * u[i];
    }
    store4<E>(static_cast<E*>(g.c) + at2, dg);
    store4<E>(static_cast<E*>(g.c) + at2 + g.N, du);
    if (g.h) store4<E>(static_cast<E*>(g.h) + at, h);
  }
}

// Workgroup tile BM x BN (kGlu: BN / 2 gate and BN / 2 up rows of B) in WM x WN
// waves; STAGES buffers of kBK.  Stage kt + STAGES goes into the buffer of stage
// kt once every wave has read it (the barrier in the last substep of step kt).
template <class E, int BM, int BN, int WM, int WN, int STAGES, bool ACOL, bool BCOL, int EPI, bool SPLIT>
__global__ __launch_bounds__(WM * WN * 64, BM == 256 ? 2 : 2) void dense_gemm_kernel(DenseGemm g, int tiles_m, int tiles_n, int splits) {
  constexpr int NW = WM * WN;
  constexpr bool DUAL = EPI == kGlu;
  constexpr int NC = DUAL ? BN / 2 : BN;  // columns of C per tile
  using A = Operand<BM, ACOL, NW, 1>;
  using B = Operand<BN, BCOL, NW, DUAL ? 2 : 1>;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static_assert(!DUAL || TN % 2 == 0, "gate and up pairs");
  constexpr int STAGE = A::kBytes + B::kBytes, N_DMA = A::kCopies + B::kCopies;
  static_assert((STAGES - 1) * N_DMA < 64, "vmcnt range");
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];

  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  // Workgroups land on the XCDs in turn: each XCD takes one contiguous range of
  // tiles, column by column over groups of eight row tiles.
  const int total = tiles_m * tiles_n * splits;
  const int per = (total + 7) / 8;
  int t = (blockIdx.x % 8) * per + blockIdx.x / 8;
  if (t >= total || static_cast<int>(blockIdx.x / 8) >= per) return;
  const int split = t / (tiles_m * tiles_n);
  t %= tiles_m * tiles_n;
  constexpr int GM = 8;
  const int grp = t / (GM * tiles_n), in = t % (GM * tiles_n), gsz = min(GM, tiles_m - grp * GM);
  const int m0 = (grp * GM + in % gsz) * BM, n0 = (in / gsz) * NC;

  const int nk_all = (g.K + kBK - 1) / kBK;
  const int kt0 = static_cast<int>(static_cast<long>(nk_all) * split / splits);
  const int nk = static_cast<int>(static_cast<long>(nk_all) * (split + 1) / splits) - kt0;
  const int k_first = kt0 * kBK;

  A a;
  B b;
  {
    const uint16_t* pa = static_cast<const uint16_t*>(g.a);
    const uint16_t* pb = static_cast<const uint16_t*>(g.b);
    if constexpr (ACOL) a.cols(pa, m0, g.M, k_first);
    else a.rows(0, pa + static_cast<size_t>(m0) * g.K, g.M - m0, g.K, k_first);
    if constexpr (BCOL) b.cols(pb, n0, g.N, k_first);
    else b.rows(0, pb + static_cast<size_t>(n0) * g.K, g.N - n0, g.K, k_first);
    if constexpr (DUAL) b.rows(1, pb + (static_cast<size_t>(g.N) + n0) * g.K, g.N - n0, g.K, k_first);
    a.offsets(wave, lane);
    b.offsets(wave, lane);
  }
  const uint32_t smem0 = lds_addr(smem);
  auto issue = [&](int kt) {
    const uint32_t buf = smem0 + (kt % STAGES) * STAGE;
    const int k = k_first + kt * kBK;
    a.issue(k, g.K, wave, lane, buf);
    b.issue(k, g.K, wave, lane, buf + A::kBytes);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x16{};
  // B row (within the tile) of wave tile j
  auto brow = [&](int j) { return DUAL ? (j < TN / 2 ? wn * (WTN / 2) + j * 32 : NC + wn * (WTN / 2) + (j - TN / 2) * 32) : wn * WTN + j * 32; };

  u32x4 fa[2][TM], fb[2][TN];
  auto read = [&](int kt, int kk, int buf) {
    const uint32_t at = smem0 + (kt % STAGES) * STAGE;
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[buf][i] = A::frag(at, wm * WTM + i * 32, kk, lane);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[buf][j] = B::frag(at + A::kBytes, brow(j), kk, lane);
  };
  // at most `ahead` later steps' copies of this wave are still in flight
  auto wait_ahead = [&](int ahead) {
    if constexpr (STAGES >= 4) { if (ahead >= 3) { vm_wait<3 * N_DMA>(); return; } }
    if constexpr (STAGES >= 3) { if (ahead == 2) { vm_wait<2 * N_DMA>(); return; } }
    if (ahead == 1) { vm_wait<N_DMA>(); return; }
    vm_wait<0>();
  };

  const int first = min(STAGES, nk);
  for (int s = 0; s < first; ++s) issue(s);
  wait_ahead(first - 1);
  bar();
  read(0, 0, 0);
  constexpr int NKK = kBK / 16;
  for (int kt = 0; kt < nk; ++kt) {
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      if (kk + 1 < NKK) {
        read(kt, kk + 1, (kk + 1) & 1);
      } else if (kt + 1 < nk) {
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        lds_wait();  // this wave holds all of stage kt in registers
        wait_ahead(min(STAGES - 2, nk - 2 - kt));
        bar();  // stage kt + 1 has landed, stage kt's buffer is free
        if (kt + STAGES < nk) issue(kt + STAGES);
        read(kt + 1, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma32<E>(fb[kk & 1][j], fa[kk & 1][i], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Lane: row m0 + .. + lane % 32, four consecutive columns per quarter of the block.
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + wm * WTM + i * 32 + (lane & 31);
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < (DUAL ? TN / 2 : TN); ++j) {
      const int nb = n0 + brow(j) + 4 * (lane >> 5);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = nb + 8 * q;
        if (n >= g.N) continue;
        f32x4 c, up{};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c[e] = acc[i][j][4 * q + e];
          if (DUAL) up[e] = acc[i][j + (DUAL ? TN / 2 : 0)][4 * q + e];
        }
        if constexpr (SPLIT) {
          const int w = DUAL ? 2 * g.N : g.N;
          float* p = g.part + (static_cast<size_t>(split) * g.M + m) * w + n;
          *reinterpret_cast<f32x4*>(p) = c;
          if (DUAL) *reinterpret_cast<f32x4*>(p + g.N) = up;
        } else {
          finish4<E, EPI>(g, m, n, c, up);
        }
      }
    }
  }
}

// The partial products of a split K, added in the order of the splits, and the epilogue.
template <class E, int EPI>
__global__ __launch_bounds__(256) void dense_join_kernel(DenseGemm g, int splits) {
  constexpr bool DUAL = EPI == kGlu;
  const size_t per_row = g.N / 4, n4 = static_cast<size_t>(g.M) * per_row;
  const int w = DUAL ? 2 * g.N : g.N;
  for (size_t i = blockIdx.x * 256ul + threadIdx.x; i < n4; i += gridDim.x * 256ul) {
    const int m = static_cast<int>(i / per_row), n = static_cast<int>(i % per_row) * 4;
    f32x4 c{}, up{};
    for (int s = 0; s < splits; ++s) {
      const float* p = g.part + (static_cast<size_t>(s) * g.M + m) * w + n;
      c += *reinterpret_cast<const f32x4*>(p);
      if (DUAL) up += *reinterpret_cast<const f32x4*>(p + g.N);
    }
    finish4<E, EPI>(g, m, n, c, up);
  }
}

namespace {

struct Plan {
  int tile;  // rows of A per tile: 256, 128 or 64
  int splits;
};

int columns_of(int tile, bool dual) { return (tile == 256 ? 256 : 128) / (dual ? 2 : 1); }

Plan plan_for(int epi, int M, int N, int K) {
  Plan p;
  const bool dual = epi == kGlu;
  p.tile = M > 1024 ? 256 : M > 64 ? 128 : 64;
  const long tiles = static_cast<long>((M + p.tile - 1) / p.tile) * ((N + columns_of(p.tile, dual) - 1) / columns_of(p.tile, dual));
  const int nk = (K + kBK - 1) / kBK;
  const long room = (p.tile == 256 ? 256 : 512) / std::max(1L, tiles);
  p.splits = static_cast<int>(std::max(1L, std::min({room, static_cast<long>(nk / 4), 16L})));
  return p;
}

template <class E, int BM, int BN, int WM, int WN, int STAGES, bool ACOL, bool BCOL, int EPI>
hipError_t run_tile(const DenseGemm& g, int splits, hipStream_t s) {
  constexpr int NC = EPI == kGlu ? BN / 2 : BN;
  constexpr int lds = STAGES * (BM + BN) * kBK * 2;
  const int tm = (g.M + BM - 1) / BM, tn = (g.N + NC - 1) / NC;
  const long total = static_cast<long>(tm) * tn * splits;
  const dim3 grid(static_cast<unsigned>((total + 7) / 8 * 8)), block(WM * WN * 64);
  auto go = [&](auto kernel) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    kernel<<<grid, block, lds, s>>>(g, tm, tn, splits);
    return hipGetLastError();
  };
  if (splits == 1) return go(dense_gemm_kernel<E, BM, BN, WM, WN, STAGES, ACOL, BCOL, EPI, false>);
  const hipError_t e = go(dense_gemm_kernel<E, BM, BN, WM, WN, STAGES, ACOL, BCOL, EPI, true>);
  if (e != hipSuccess) return e;
  const size_t n4 = static_cast<size_t>(g.M) * (g.N / 4);
  dense_join_kernel<E, EPI><<<static_cast<unsigned>(std::min<size_t>((n4 + 255) / 256, 2048)), 256, 0, s>>>(g, splits);
  return hipGetLastError();
}

template <class E, bool ACOL, bool BCOL, int EPI>
hipError_t run(const DenseGemm& g, hipStream_t s) {
  const Plan p = plan_for(EPI, g.M, g.N, g.K);
  if (p.tile == 256) return run_tile<E, 256, 256, 2, 4, 2, ACOL, BCOL, EPI>(g, p.splits, s);
  if (p.tile == 128) return run_tile<E, 128, 128, 2, 2, 2, ACOL, BCOL, EPI>(g, p.splits, s);
  return run_tile<E, 64, 128, 2, 2, 3, ACOL, BCOL, EPI>(g, p.splits, s);
}

template <class E>
hipError_t run_type(int layout, int epi, const DenseGemm& g, hipStream_t s) {
  if (layout == kRowRow && epi == kGlu) return run<E, false, false, kGlu>(g, s);
  if (layout == kRowRow && epi == kStore) return run<E, false, false, kStore>(g, s);
  if (layout == kRowCol && epi == kDglu) return run<E, false, true, kDglu>(g, s);
  if (layout == kRowCol && epi == kStore) return run<E, false, true, kStore>(g, s);
  if (layout == kColCol && epi == kStore) return run<E, true, true, kStore>(g, s);
  return hipErrorInvalidValue;
}

}  // namespace

size_t dense_gemm_workspace_bytes(int, int epi, int M, int N, int K) {
  const Plan p = plan_for(epi, M, N, K);
  return p.splits == 1 ? 0 : static_cast<size_t>(p.splits) * M * N * (epi == kGlu ? 2 : 1) * 4;
}

hipError_t launch_dense_gemm(int dtype, int layout, int epi, const DenseGemm& g, hipStream_t s) {
  return dtype == kBf16 ? run_type<bf16_t>(layout, epi, g, s) : run_type<f16_t>(layout, epi, g, s);
}

}  // namespace moe
