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
// The four wait states between the write of M0 and the copy (one is needed for M0)
// also cover a descriptor word that the compiler took from a VGPR just before.
__device__ __forceinline__ void bdma16(const u32x4& rsrc, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc)
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

  uint64_t base[PARTS];  // where the next step starts
  int left[PARTS];       // row: bytes from there to the end of the tile's rows; column: bytes before it in its row
  uint32_t voff[kCopies];
  u32x4 desc[PARTS];     // the step being copied
  uint32_t past;         // row: all ones above the offsets where the lane's chunk lies past K
  int ld, chunk;

  // row operand: `at` the first of `rows` rows that exist from the tile's start
  __device__ void rows(int part, const void* at, int rows, int ld_, int k0) {
    ld = ld_;
    base[part] = reinterpret_cast<uint64_t>(at) + static_cast<uint64_t>(k0) * 2;
    left[part] = __builtin_amdgcn_readfirstlane(max(0, max(0, min(rows, R / PARTS)) * ld_ * 2 - k0 * 2));
  }
  // column operand: column m0 of the rows from k0 on
  __device__ void cols(const void* at, int m0, int ld_, int k0) {
    ld = ld_;
    base[0] = reinterpret_cast<uint64_t>(at) + (static_cast<uint64_t>(k0) * ld_ + m0) * 2;
    left[0] = __builtin_amdgcn_readfirstlane(m0 * 2);
  }
  __device__ void offsets(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = ((i % (kCopies / PARTS)) * NW + wave) * kRows + lane / kChunks;  // row within its part
      const int c = (lane % kChunks) ^ (COL ? tswz(r) : (r >> 1) & 7);
      if (i == 0) chunk = c;
      voff[i] = static_cast<uint32_t>(r) * static_cast<uint32_t>(ld) * 2u + c * 16u;
    }
    static_assert(COL || NW % 2 == 0, "a lane's chunk is the same in every copy");
  }
  // Make ready for the step that starts at k (of K; past its end the copies
  // are zeros), and stand at the next one.
  __device__ void step(int k, int K) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      desc[p] = buffer_of(base[p], COL ? max(0, max(0, min(K - k, kBK)) * ld * 2 - left[p]) : left[p]);
      base[p] += COL ? static_cast<uint64_t>(ld) * kBK * 2 : kBK * 2;
      if (!COL) left[p] = max(0, left[p] - kBK * 2);
    }
    if (!COL) past = k + chunk * 8 >= K ? 0x80000000u : 0u;
  }
  // Copy i of that step into LDS at `lds`.
  __device__ void copy(int i, int wave, uint32_t lds) const {
    bdma16(desc[i / (kCopies / PARTS)], COL ? voff[i] : voff[i] | past, lds + (i * NW + wave) * 1024);
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

// What an epilogue reads beside the products, for eight columns of one row.
template <class E, int EPI> struct Beside {
  f32x8 p, q;
  __device__ void load(const DenseGemm& g, int m, int n) {
    if constexpr (EPI == kStore) {
      if (g.add) p = load8<E>(static_cast<const E*>(g.add) + static_cast<size_t>(m) * g.N + n);
    } else if constexpr (EPI == kDglu) {
      const float* at = g.pre_in + static_cast<size_t>(m) * 2 * g.N + n;
      p = load8<float>(at);
      q = load8<float>(at + g.N);
    }
  }
};

// The epilogue on eight columns of one row.
template <class E, int EPI>
__device__ __forceinline__ void finish8(const DenseGemm& g, int m, int n, const f32x8& c, const f32x8& up, const Beside<E, EPI>& x) {
  const size_t at = static_cast<size_t>(m) * g.N + n;
  const size_t at2 = static_cast<size_t>(m) * 2 * g.N + n;
  if constexpr (EPI == kStore) {
    store8<E>(static_cast<E*>(g.c) + at, g.add ? c + x.p : c);
  } else if constexpr (EPI == kGlu) {
    if (g.pre) {
      store8<float>(g.pre + at2, c);
      store8<float>(g.pre + at2 + g.N, up);
    }
    f32x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = act_of(g.act, c[i]) * up[i];
    store8<E>(static_cast<E*>(g.c) + at, h);
  } else {
    f32x8 dg, du, h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a, da;
      act_and_slope(g.act, x.p[i], a, da);
      dg[i] = c[i] * x.q[i] * da;
      du[i] = c[i] * a;
      h[i] = a * x.q[i];
    }
    store8<E>(static_cast<E*>(g.c) + at2, dg);
    store8<E>(static_cast<E*>(g.c) + at2 + g.N, du);
    if (g.h) store8<E>(static_cast<E*>(g.h) + at, h);
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
  const int k_first = kt0 * kBK, k_end = min(g.K, k_first + nk * kBK);

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
  // Copies [from, to) of stage kt: A's, then B's.
  auto ready = [&](int kt) {
    a.step(k_first + kt * kBK, k_end);
    b.step(k_first + kt * kBK, k_end);
  };
  auto copy = [&](int i, uint32_t buf) {
    if (i < A::kCopies) a.copy(i, wave, buf);
    else b.copy(i - A::kCopies, wave, buf + A::kBytes);
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x16{};
  // B row (within the tile) of wave tile j
  auto brow = [&](int j) { return DUAL ? (j < TN / 2 ? wn * (WTN / 2) + j * 32 : NC + wn * (WTN / 2) + (j - TN / 2) * 32) : wn * WTN + j * 32; };

  u32x4 fa[2][TM], fb[2][TN];
  auto read = [&](uint32_t at, int kk, int buf) {
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[buf][i] = A::frag(at, wm * WTM + i * 32, kk, lane);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[buf][j] = B::frag(at + A::kBytes, brow(j), kk, lane);
  };
  // The products of one substep, with copies [from, from + COUNT) spread between them.
  auto multiply = [&](int buf, auto from, auto count, uint32_t dst) {
    constexpr int FROM = decltype(from)::value, COUNT = decltype(count)::value, EVERY = COUNT ? (TM * TN + COUNT - 1) / COUNT : 1;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int n = i * TN + j;
        acc[i][j] = mfma32<E>(fb[buf][j], fa[buf][i], acc[i][j]);
        if (n % EVERY == EVERY - 1 && n / EVERY < COUNT) {
          __builtin_amdgcn_sched_barrier(0);
          copy(FROM + n / EVERY, dst);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
    for (int c = TM * TN / EVERY; c < COUNT; ++c) copy(FROM + c, dst);
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int NKK = kBK / 16, HALF = N_DMA / 2;
  static_assert(NKK == 4 && N_DMA % 2 == 0, "substeps");
  using std::integral_constant;
  typedef integral_constant<int, 0> zero;
  typedef integral_constant<int, HALF> half;

  // Stages 0 .. STAGES - 2 whole and half of the next; from then on each step
  // copies the other half of its stage kt + STAGES - 1 and the first of the
  // next.  Steps past the end copy zeros, so every wait counts the same.
  uint32_t rd = smem0, wr = smem0;  // the buffers of stage kt and of the stage being copied
  auto next = [&](uint32_t at) { return at + STAGE == smem0 + STAGES * STAGE ? smem0 : at + STAGE; };
#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
    ready(s);
#pragma unroll
    for (int i = 0; i < (s < STAGES - 1 ? N_DMA : HALF); ++i) copy(i, wr);
    if (s < STAGES - 1) wr = next(wr);
  }
  vm_wait<(STAGES - 2) * N_DMA + HALF>();
  bar();
  read(rd, 0, 0);
  for (int kt = 0; kt < nk; ++kt) {
    read(rd, 1, 1);
    __builtin_amdgcn_sched_barrier(0);
    multiply(0, half{}, half{}, wr);
    read(rd, 2, 0);
    __builtin_amdgcn_sched_barrier(0);
    multiply(1, zero{}, zero{}, wr);
    read(rd, 3, 1);
    __builtin_amdgcn_sched_barrier(0);
    multiply(0, zero{}, zero{}, wr);
    ready(kt + STAGES);
    wr = rd;
    rd = next(rd);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    lds_wait();  // this wave holds all of stage kt in registers
    vm_wait<(STAGES - 2) * N_DMA>();
    bar();  // stage kt + 1 has landed, stage kt's buffer is free
    read(rd, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    multiply(1, zero{}, half{}, wr);
  }
  vm_wait<0>();

  // A wave turns its 32-row blocks over in LDS of its own, so that every load
  // and store of the epilogue takes whole lines: eight columns per lane.
  constexpr int PITCH = WTN + 4;  // floats per row: sixteen lanes' 16-byte writes lie in different banks
  static_assert(NW * 32 * PITCH * 4 <= STAGES * STAGE, "the epilogue's rows fit the stages");
  constexpr int LPR = WTN / (DUAL ? 16 : 8), RPI = 64 / LPR;  // lanes per row, rows per pass
  bar();  // no wave reads the stages any more
  float* const mine = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
  const int er = lane / LPR, ec = lane % LPR * 8;
  const int n = n0 + (DUAL ? wn * (WTN / 2) : wn * WTN) + ec;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int mb = m0 + wm * WTM + i * 32 + er;
    Beside<E, EPI> x[32 / RPI];
    if (!SPLIT && n < g.N) {
#pragma unroll
      for (int r = 0; r < 32 / RPI; ++r)
        if (mb + r * RPI < g.M) x[r].load(g, mb + r * RPI, n);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
        *reinterpret_cast<f32x4*>(mine + (lane & 31) * PITCH + j * 32 + 8 * q + 4 * (lane >> 5)) = v;
      }
#pragma unroll
    for (int r = 0; r < 32 / RPI; ++r) {
      const int m = mb + r * RPI;
      if (m >= g.M || n >= g.N) continue;
      const float* row = mine + (r * RPI + er) * PITCH + ec;
      const f32x8 c = load8<float>(row);
      f32x8 up{};
      if constexpr (DUAL) up = load8<float>(row + WTN / 2);
      if constexpr (SPLIT) {
        const int w = DUAL ? 2 * g.N : g.N;
        float* p = g.part + (static_cast<size_t>(split) * g.M + m) * w + n;
        store8<float>(p, c);
        if (DUAL) store8<float>(p + g.N, up);
      } else {
        finish8<E, EPI>(g, m, n, c, up, x[r]);
      }
    }
  }
}

// The partial products of a split K, added in the order of the splits, and the epilogue.
template <class E, int EPI>
__global__ __launch_bounds__(256) void dense_join_kernel(DenseGemm g, int splits) {
  constexpr bool DUAL = EPI == kGlu;
  const size_t per_row = g.N / 8, n8 = static_cast<size_t>(g.M) * per_row;
  const int w = DUAL ? 2 * g.N : g.N;
  for (size_t i = blockIdx.x * 256ul + threadIdx.x; i < n8; i += gridDim.x * 256ul) {
    const int m = static_cast<int>(i / per_row), n = static_cast<int>(i % per_row) * 8;
    Beside<E, EPI> x;
    x.load(g, m, n);
    f32x8 c{}, up{};
    for (int s = 0; s < splits; ++s) {
      const float* p = g.part + (static_cast<size_t>(s) * g.M + m) * w + n;
      c += load8<float>(p);
      if (DUAL) up += load8<float>(p + g.N);
    }
    finish8<E, EPI>(g, m, n, c, up, x);
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
  const size_t n8 = static_cast<size_t>(g.M) * (g.N / 8);
  dense_join_kernel<E, EPI><<<static_cast<unsigned>(std::min<size_t>((n8 + 255) / 256, 2048)), 256, 0, s>>>(g, splits);
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
