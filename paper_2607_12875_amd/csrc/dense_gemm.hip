// The products of the gated feed-forward block (a shared expert beside the
// routed ones, or a dense layer), 16-bit operands and fp32 sums on
// v_mfma_f32_32x32x16:
//   forward   pre = x W1^T -> h = act(gate) * up in the epilogue;  y = h W2^T (+ add)
//   backward  dh = dy W2 -> dpre = [dh u act'(g), dh act(g)] and h in the epilogue;
//             dx = dpre W1;  dW1 = dpre^T x;  dW2 = dy^T h
// Four tile kernels, of 64 x 64 to 256 x 256, take each of the six: an operand lies in
// memory with its reduction index innermost (a row operand) or outermost (a column
// operand), and goes to LDS as it lies.  A fragment of a row operand is one ds_read_b128; of a column
// operand two ds_read_b64_tr_b16, which transpose 4 x 16 blocks on the way.
#include <algorithm>
#include <utility>

#include "common.hpp"
#include "dense.hpp"
#include "dense_finish.hpp"
#include "dense_math.hpp"
#include "lds_dma.hpp"

namespace moe {

constexpr int kBK = 64;  // K elements per step: 128 bytes, one line of a row operand

// Sixteen bytes per lane from a bounds-checked buffer to LDS: lane l reads
// offset voff + soff and lands at lds + AT + 16 l.  Lanes past the buffer's end
// write zeros.  One wait state lies between the write of M0 and the copy; that the
// descriptor's words are not written by a VALU operation in the five states before
// is up to the caller, who makes them some products ahead.
template <int AT>
__device__ __forceinline__ void bdma16(const u32x4& rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %4 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc), "i"(AT), "s"(soff)
               : "memory", "m0", "scc");
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

  // Row operand: the buffer is the tile's rows, whole, and a step's place in K an
  // offset that all lanes share; rows past the last lie past the buffer's end, and
  // in the last step of a ragged K the lanes past K are sent there.  Column operand:
  // the buffer is the step's rows of K, so that those past K lie past its end.
  u32x4 desc[PARTS];
  uint32_t voff[kCopies], soff;
  uint64_t base;          // column: where the next step starts
  uint32_t whole, tail;   // column: bytes of a whole step's buffer and of a last, ragged one
  int ld, chunk;

  // The R rows (columns) from r0 on of an operand that has `count` of them, from
  // k0 of K on.  Two parts: R / 2 from r0 and R / 2 from apart + r0 on.
  __device__ void start(const void* at, int r0, int count, int K, int k0, int apart) {
    const uint64_t first = reinterpret_cast<uint64_t>(at);
    ld = COL ? count : K;
    soff = 0;
    if constexpr (COL) {
      base = first + (static_cast<uint64_t>(k0) * ld + r0) * 2;
      whole = (static_cast<uint32_t>(kBK) * ld - r0) * 2u;
      tail = K % kBK ? (static_cast<uint32_t>(K % kBK) * ld - r0) * 2u : whole;
    } else {
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
        desc[p] = buffer_of(first + static_cast<uint64_t>(r0 + p * apart) * ld * 2, static_cast<uint32_t>(max(0, min(count - r0, R / PARTS))) * ld * 2u);
    }
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
  // Make ready for the step that starts at k (of K; past its end the copies are
  // zeros).  Steps come in order.
  __device__ void step(int k, int K) {
    if constexpr (COL) {
      desc[0] = buffer_of(base, k + kBK <= K ? whole : k < K ? tail : 0u);
      base += static_cast<uint64_t>(ld) * kBK * 2;
    } else {
      // past the end the offset stays zero: the bounds check takes it off the
      // buffer's length, which one row's buffer would not have left
      soff = k < K ? k * 2u : 0u;
      if (k + kBK > K) {  // uniform
#pragma unroll
        for (int i = 0; i < kCopies; ++i) voff[i] = k + chunk * 8 >= K ? 0x80000000u : voff[i];
      }
    }
  }
  // Copy I of that step into LDS at `lds`, the buffer plus 1 KB per wave.
  template <int I> __device__ void copy(uint32_t lds) const {
    bdma16<I * NW * 1024>(desc[I / (kCopies / PARTS)], voff[I], soff, lds);
  }

  // Fragments, eight consecutive k of group lane / 32 of a K substep for row
  // lane % 32 of a block of 32 rows: where this lane reads in a buffer, for the four
  // substeps (row operand) or the four blocks from row r0 on (column operand; r0 a
  // multiple of 128 where there are four), the rest is a constant.
  __device__ static void lanes(uint32_t (&at)[4], int r0, int lane) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (!COL) {
        const int r = r0 + (lane & 31);
        at[q] = r * 128 + (((2 * q + (lane >> 5)) ^ ((r >> 1) & 7)) << 4);
      } else {
        // lane group of 16: columns 16 ((lane >> 4) & 1) .. of the block, rows 8 (lane >> 5) ..
        const int k = (lane & 15) >> 2;  // and k + 4
        const int c = r0 / 8 + 4 * q + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        at[q] = (8 * (lane >> 5) + k) * (R * 2) + ((c ^ tswz(k)) << 4) + ((lane & 1) << 3);
      }
    }
  }
  // Block `i` (rows apart: `rows`) at substep kk; at[] with the buffer's address added.
  __device__ static u32x4 frag(const uint32_t (&at)[4], int i, int rows, int kk) {
    if constexpr (!COL) {
      return lds16(at[kk] + rows * 128);
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* lp;
      const uint32_t p = at[i] + 16 * kk * (R * 2);
      const i32x2 lo = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p));
      const i32x2 hi = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * R * 2)));
      return u32x4{static_cast<uint32_t>(lo.x), static_cast<uint32_t>(lo.y), static_cast<uint32_t>(hi.x),
                   static_cast<uint32_t>(hi.y)};
    }
  }
};

// f(integral_constant<int, 0>) .. f(integral_constant<int, N - 1>)
template <class F, int... I>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void each(F f) { each(std::make_integer_sequence<int, N>{}, f); }

// The part of the product that a workgroup computes.
struct Place {
  int m0, n0, split, k_first, k_end, nk;
};
// Workgroups land on the XCDs in turn: each XCD takes one contiguous range of
// tiles, column by column over groups of eight row tiles.  False: nothing left.
template <int BM, int NC>
__device__ __forceinline__ bool place_of(const DenseGemm& g, int tiles_m, int tiles_n, int splits, Place& p) {
  const int total = tiles_m * tiles_n * splits;
  const int per = (total + 7) / 8;
  int t = (blockIdx.x % 8) * per + blockIdx.x / 8;
  if (t >= total || static_cast<int>(blockIdx.x / 8) >= per) return false;
  p.split = t / (tiles_m * tiles_n);
  t %= tiles_m * tiles_n;
  constexpr int GM = 8;
  const int grp = t / (GM * tiles_n), in = t % (GM * tiles_n), gsz = min(GM, tiles_m - grp * GM);
  p.m0 = (grp * GM + in % gsz) * BM;
  p.n0 = (in / gsz) * NC;
  const int nk_all = (g.K + kBK - 1) / kBK;
  const int kt0 = static_cast<int>(static_cast<long>(nk_all) * p.split / splits);
  p.nk = static_cast<int>(static_cast<long>(nk_all) * (p.split + 1) / splits) - kt0;
  p.k_first = kt0 * kBK;
  p.k_end = min(g.K, p.k_first + p.nk * kBK);
  return true;
}

// The waves of a tile: WM x WN of them, TM x TN blocks of 32 x 32 each.
template <int BM, int BN, int WM, int WN, int EPI> struct Waves {
  static constexpr bool DUAL = EPI == kGlu;
  static constexpr int NW = WM * WN, NC = DUAL ? BN / 2 : BN;  // NC: columns of C per tile
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static_assert(!DUAL || TN % 2 == 0, "gate and up pairs");
  static constexpr int PITCH = WTN + 4;  // floats per row of the epilogue: sixteen lanes' 16-byte writes lie in different banks
  static constexpr int kEpilogueBytes = NW * 32 * PITCH * 4;
  // first B row of wave column wn, and the rows from there to its block j
  __device__ static int bfirst(int wn) { return wn * (DUAL ? WTN / 2 : WTN); }
  __device__ static constexpr int brows(int j) { return DUAL && j >= TN / 2 ? NC + (j - TN / 2) * 32 : j * 32; }
};

// A wave turns its 32-row blocks over in LDS of its own, so that every load and
// store of the epilogue takes whole lines: eight columns per lane.
template <class E, class W, int EPI, bool SPLIT>
__device__ __forceinline__ void epilogue(const DenseGemm& g, const Place& p, int wm, int wn, int lane, float* mine,
                                         const f32x16 (&acc)[W::TM][W::TN]) {
  constexpr bool DUAL = W::DUAL;
  constexpr int PITCH = W::PITCH, WTN = W::WTN;
  constexpr int LPR = WTN / (DUAL ? 16 : 8), RPI = 64 / LPR;  // lanes per row, rows per pass
  const int er = lane / LPR, ec = lane % LPR * 8;
  const int n = p.n0 + (DUAL ? wn * (WTN / 2) : wn * WTN) + ec;
#pragma unroll
  for (int i = 0; i < W::TM; ++i) {
    const int mb = p.m0 + wm * W::WTM + i * 32 + er;
    Beside<E, EPI> x[32 / RPI];
    if (!SPLIT && n < g.N) {
#pragma unroll
      for (int r = 0; r < 32 / RPI; ++r)
        if (mb + r * RPI < g.M) x[r].load(g, mb + r * RPI, n);
    }
#pragma unroll
    for (int j = 0; j < W::TN; ++j)
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
        float* at = g.part + (static_cast<size_t>(p.split) * g.M + m) * w + n;
        store8<float>(at, c);
        if (DUAL) store8<float>(at + g.N, up);
      } else {
        finish8<E, EPI>(g, m, n, c, up, x[r]);
      }
    }
  }
}

// A wave's fragments, for this K substep and the next, and its products.
template <class E, class W, class A, class B> struct Math {
  static constexpr int TM = W::TM, TN = W::TN, N = TM * TN, R = TM + TN;
  u32x4 fa[2][TM], fb[2][TN];
  f32x16 acc[TM][TN];
  uint32_t la[4], lb[4], pa[4], pb[4];  // where the lane reads in a buffer, and in the buffers being read
  __device__ void start(int a0, int b0, int lane) {
    A::lanes(la, a0, lane);
    B::lanes(lb, b0, lane);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = f32x16{};
  }
  __device__ void from(uint32_t at_a, uint32_t at_b) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      pa[q] = la[q] + at_a;
      pb[q] = lb[q] + at_b;
    }
  }
  // fragment r of substep kk, in the order that the products want them
  __device__ void read(int kk, int r) {
    if (r < TN) fb[kk & 1][r] = B::frag(pb, r, W::brows(r), kk);
    else fa[kk & 1][r - TN] = A::frag(pa, r - TN, (r - TN) * 32, kk);
  }
  __device__ void read(int kk) {
#pragma unroll
    for (int r = 0; r < R; ++r) read(kk, r);
    __builtin_amdgcn_sched_barrier(0);
  }
  // substep kk's products; work(n) after the nth
  template <class F> __device__ void multiply(int kk, F work) {
    each<N>([&](auto n) {
      constexpr int i = n / TN, j = n % TN;
      acc[i][j] = mfma32<E>(fb[kk & 1][j], fa[kk & 1][i], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
      work(n);
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  __device__ void multiply(int kk) {
#pragma unroll
    for (int n = 0; n < N; ++n) acc[n / TN][n % TN] = mfma32<E>(fb[kk & 1][n % TN], fa[kk & 1][n / TN], acc[n / TN][n % TN]);
    __builtin_amdgcn_sched_barrier(0);
  }
};

// Before a barrier that frees a buffer: this wave's fragments of it have arrived,
// and at most N of its copies are still in flight.
template <int N>
__device__ __forceinline__ void settle() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  lds_wait();
  vm_wait<N>();
}

// 128 x 128 tile (kGlu: 64 gate and 64 up rows of B), four waves of 64 x 64; STAGES
// buffers of kBK.  Stage kt + STAGES goes into the buffer of stage
// kt once every wave has read it (the barrier before the last substep of step
// kt): half of its copies in that substep, half in the next.  Steps past the end
// copy zeros, so there is no branch in the loop and every wait counts the same.
template <class E, int STAGES, bool ACOL, bool BCOL, int EPI, bool SPLIT>
__global__ __launch_bounds__(256, 2) void dense_gemm_128_kernel(DenseGemm g, int tiles_m, int tiles_n, int splits) {
  constexpr int BM = 128, BN = 128, WM = 2, WN = 2;
  using W = Waves<BM, BN, WM, WN, EPI>;
  using A = Operand<BM, ACOL, W::NW, 1>;
  using B = Operand<BN, BCOL, W::NW, W::DUAL ? 2 : 1>;
  constexpr int STAGE = A::kBytes + B::kBytes, N_DMA = A::kCopies + B::kCopies, HALF = N_DMA / 2;
  static_assert(N_DMA % 2 == 0 && (STAGES - 1) * N_DMA < 64 && W::kEpilogueBytes <= STAGES * STAGE, "stages");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[STAGES * STAGE];

  Place p;
  if (!place_of<BM, W::NC>(g, tiles_m, tiles_n, splits, p)) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  A a;
  B b;
  a.start(g.a, p.m0, g.M, g.K, p.k_first, 0);
  b.start(g.b, p.n0, g.N, g.K, p.k_first, g.N);
  a.offsets(wave, lane);
  b.offsets(wave, lane);
  auto ready = [&](int kt) {
    a.step(p.k_first + kt * kBK, p.k_end);
    b.step(p.k_first + kt * kBK, p.k_end);
  };
  const uint32_t smem0 = lds_addr(smem), mine = wave * 1024;
  auto copy = [&](auto i, uint32_t buf) {
    if constexpr (i < A::kCopies) a.template copy<i>(buf + mine);
    else b.template copy<i - A::kCopies>(buf + A::kBytes + mine);
  };
  uint32_t rd = smem0, wr = smem0;  // the buffers of stage kt and of the stage being copied
  auto next = [&](uint32_t at) { return at + STAGE == smem0 + STAGES * STAGE ? smem0 : at + STAGE; };
  Math<E, W, A, B> x;
  x.start(wm * W::WTM, W::bfirst(wn), lane);
  // copies FROM .. FROM + HALF - 1 spread over a substep's products
  auto spread = [&](int kk, auto from) {
    constexpr int EVERY = (x.N + HALF - 1) / HALF;
    x.multiply(kk, [&](auto n) {
      if constexpr (n % EVERY == EVERY - 1 && n / EVERY < HALF) copy(std::integral_constant<int, from + n / EVERY>{}, wr);
      if constexpr (n == x.N - 1)
        each<HALF>([&](auto c) {
          if constexpr (c >= x.N / EVERY) copy(std::integral_constant<int, from + c>{}, wr);
        });
    });
  };
  typedef std::integral_constant<int, 0> first_half;
  typedef std::integral_constant<int, HALF> second_half;

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    ready(s);
    each<N_DMA>([&](auto i) { copy(i, wr); });
    wr = next(wr);
  }
  ready(STAGES - 1);
  each<HALF>([&](auto i) { copy(i, wr); });
  vm_wait<(STAGES - 2) * N_DMA + HALF>();
  bar();
  x.from(rd, rd + A::kBytes);
  x.read(0);
  for (int kt = 0; kt < p.nk; ++kt) {
    x.read(1);
    spread(0, second_half{});
    x.read(2);
    x.multiply(1);
    x.read(3);
    x.multiply(2);
    ready(kt + STAGES);
    wr = rd;
    rd = next(rd);
    x.from(rd, rd + A::kBytes);
    settle<(STAGES - 2) * N_DMA>();
    bar();  // stage kt + 1 has landed, stage kt's buffer is free
    x.read(0);
    spread(3, first_half{});
  }
  vm_wait<0>();
  bar();  // no wave reads the stages any more, no copy is under way
  epilogue<E, W, EPI, SPLIT>(g, p, wm, wn, lane, reinterpret_cast<float*>(smem) + wave * 32 * W::PITCH, x.acc);
}

// 64 x 128 or 64 x 64 tile (the small one where there are few), four waves of 32 x 64
// or 32 x 32, three buffers of kBK.  A wave's substep has one or two products, 32 or 64
// cycles, fewer than an LDS read takes, so the fragments of a whole
// step are read during the step before (512 x 2048 x 1408: 8.8 us, one substep ahead
// 10.8; 128 x 7168 x 2048 11.2 and 14.0).  A stage's buffer is free once every wave
// has its fragments, at the barrier that opens its step, and stage kt + 3 goes there.
template <class E, int BN, bool ACOL, bool BCOL, int EPI, bool SPLIT>
__global__ __launch_bounds__(256, 2) void dense_gemm_64_kernel(DenseGemm g, int tiles_m, int tiles_n, int splits) {
  constexpr int BM = 64, WM = 2, WN = 2, STAGES = 3;
  using W = Waves<BM, BN, WM, WN, EPI>;
  using A = Operand<BM, ACOL, W::NW, 1>;
  using B = Operand<BN, BCOL, W::NW, W::DUAL ? 2 : 1>;
  constexpr int STAGE = A::kBytes + B::kBytes, N_DMA = A::kCopies + B::kCopies;
  constexpr int TM = W::TM, TN = W::TN, R = TM + TN, NKK = kBK / 16, N = TM * TN * NKK;
  static_assert((STAGES - 1) * N_DMA < 64 && W::kEpilogueBytes <= STAGES * STAGE, "stages");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[STAGES * STAGE];

  Place p;
  if (!place_of<BM, W::NC>(g, tiles_m, tiles_n, splits, p)) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  A a;
  B b;
  a.start(g.a, p.m0, g.M, g.K, p.k_first, 0);
  b.start(g.b, p.n0, g.N, g.K, p.k_first, g.N);
  a.offsets(wave, lane);
  b.offsets(wave, lane);
  auto ready = [&](int kt) {
    a.step(p.k_first + kt * kBK, p.k_end);
    b.step(p.k_first + kt * kBK, p.k_end);
  };
  const uint32_t smem0 = lds_addr(smem), mine = wave * 1024;
  auto copy = [&](auto i, uint32_t buf) {
    if constexpr (i < A::kCopies) a.template copy<i>(buf + mine);
    else b.template copy<i - A::kCopies>(buf + A::kBytes + mine);
  };
  auto next = [&](uint32_t at) { return at + STAGE == smem0 + STAGES * STAGE ? smem0 : at + STAGE; };

  u32x4 fa[2][NKK][TM], fb[2][NKK][TN];
  f32x16 acc[TM][TN];
  uint32_t la[4], lb[4], pa[4], pb[4];
  A::lanes(la, wm * W::WTM, lane);
  B::lanes(lb, W::bfirst(wn), lane);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x16{};
  auto from = [&](uint32_t at) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      pa[q] = la[q] + at;
      pb[q] = lb[q] + at + A::kBytes;
    }
  };
  // fragment f of a step, in the order that the products want them, into set s
  auto read = [&](auto s, auto f) {
    constexpr int kk = f / R, r = f % R;
    if constexpr (r < TN) fb[s][kk][r] = B::frag(pb, r, W::brows(r), kk);
    else fa[s][kk][r - TN] = A::frag(pa, r - TN, (r - TN) * 32, kk);
  };
  uint32_t rd = smem0;  // the buffer of stage kt
  // One step: set s multiplied, the other read from stage kt + 1, stage kt + STAGES
  // copied over stage kt, spread over the products.
  auto step = [&](auto s, int kt) {
    constexpr int WORK = NKK * R + N_DMA;
    const uint32_t wr = rd;
    rd = next(rd);
    from(rd);
    ready(kt + STAGES);
    settle<(STAGES - 2) * N_DMA>();
    bar();  // stage kt + 1 has landed, stage kt is in registers everywhere
    each<N>([&](auto n) {
      constexpr int kk = n / (TM * TN), i = n % (TM * TN) / TN, j = n % TN;
      acc[i][j] = mfma32<E>(fb[s][kk][j], fa[s][kk][i], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
      constexpr int w0 = n * WORK / N, w1 = (n + 1) * WORK / N;
      each<w1 - w0>([&](auto w) {
        constexpr int at = (w0 + w + NKK * R) % WORK;  // copies first
        if constexpr (at < NKK * R) read(std::integral_constant<int, 1 - s>{}, std::integral_constant<int, at>{});
        else copy(std::integral_constant<int, at - NKK * R>{}, wr);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  uint32_t wr = smem0;
#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
    ready(s);
    each<N_DMA>([&](auto i) { copy(i, wr); });
    wr = next(wr);
  }
  vm_wait<(STAGES - 1) * N_DMA>();
  bar();
  from(rd);
  typedef std::integral_constant<int, 0> even;
  typedef std::integral_constant<int, 1> odd;
  each<NKK * R>([&](auto f) { read(even{}, f); });
  for (int kt = 0; kt < p.nk; kt += 2) {
    step(even{}, kt);
    if (kt + 1 < p.nk) step(odd{}, kt + 1);
  }
  vm_wait<0>();
  bar();  // no wave reads the stages any more, no copy is under way
  epilogue<E, W, EPI, SPLIT>(g, p, wm, wn, lane, reinterpret_cast<float*>(smem) + wave * 32 * W::PITCH, acc);
}

// 256 x 256 tile, four waves of 128 x 128, each with a SIMD to itself (the sums
// take half of its 512 registers).  The LDS reads of the products are the fewest
// that way, 128 KB per step; with the 64 KB that land they take most of the LDS's
// time, so they are spread evenly: after a substep's sixteen products come, in
// turn, a fragment of the next substep and, every fourth time, a copy or two.  A has
// two buffers, B three, all of the 160 KB: A's eight copies follow the barrier that
// frees their buffer, in the step's last quarter, B's, for a stage further on, come
// in the half step after, none in the third quarter, so that no copy has less than
// three quarters of a step to land.  8192 tokens, 4096 x
// 11264: y = h W2^T runs the matrix pipe 78 % of the cycles (67 with eight waves of
// 128 x 64 in two groups half a step apart, 61 with eight in step), dx 79 %.
template <class E, bool ACOL, bool BCOL, int EPI, bool SPLIT>
__global__ __launch_bounds__(256, 1) void dense_gemm_256_kernel(DenseGemm g, int tiles_m, int tiles_n, int splits) {
  using W = Waves<256, 256, 2, 2, EPI>;
  using A = Operand<256, ACOL, 4, 1>;
  using B = Operand<256, BCOL, 4, W::DUAL ? 2 : 1>;
  constexpr int NA = A::kCopies, NB = B::kCopies;
  static_assert(NA == 8 && NB == 8 && W::kEpilogueBytes <= 2 * A::kBytes + 3 * B::kBytes, "eight copies each");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * A::kBytes + 3 * B::kBytes];

  Place p;
  if (!place_of<256, W::NC>(g, tiles_m, tiles_n, splits, p)) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / 2, wn = wave % 2;
  A a;
  B b;
  a.start(g.a, p.m0, g.M, g.K, p.k_first, 0);
  b.start(g.b, p.n0, g.N, g.K, p.k_first, g.N);
  a.offsets(wave, lane);
  b.offsets(wave, lane);
  const uint32_t a0 = lds_addr(smem), b0 = a0 + 2 * A::kBytes, mine = wave * 1024;
  uint32_t ra = a0, rb = b0, wa = a0, wb = b0;  // buffers being read and written
  auto next_a = [&](uint32_t at) { return at == a0 ? a0 + A::kBytes : a0; };
  auto next_b = [&](uint32_t at) { return at == b0 + 2 * B::kBytes ? b0 : at + B::kBytes; };
  auto ready_a = [&](int kt) { a.step(p.k_first + kt * kBK, p.k_end); };
  auto ready_b = [&](int kt) { b.step(p.k_first + kt * kBK, p.k_end); };
  Math<E, W, A, B> x;
  x.start(wm * W::WTM, W::bfirst(wn), lane);
  // substep kk, the next one's fragments, and copy(0) .. copy(3)
  auto substep = [&](int kk, auto copy) {
    x.multiply(kk, [&](auto n) {
      if constexpr (n % 2 == 0) x.read((kk + 1) % 4, n / 2);
      else if constexpr (n % 4 == 1) copy(std::integral_constant<int, n / 4>{});
    });
  };
  auto a_both = [&](auto c) {
    a.template copy<c>(wa + mine);
    a.template copy<c + 4>(wa + mine);
  };
  auto b_low = [&](auto c) { b.template copy<c>(wb + mine); };
  auto b_high = [&](auto c) { b.template copy<c + 4>(wb + mine); };

  // stages 0 and 1, B first; then B's stage 2 before A's, as in the loop
  ready_b(0);
  each<NB>([&](auto i) { b.template copy<i>(wb + mine); });
  wb = next_b(wb);
  ready_a(0);
  each<NA>([&](auto i) { a.template copy<i>(wa + mine); });
  wa = next_a(wa);
  ready_b(1);
  each<NB>([&](auto i) { b.template copy<i>(wb + mine); });
  wb = next_b(wb);
  ready_a(1);
  each<NA>([&](auto i) { a.template copy<i>(wa + mine); });
  vm_wait<NA + NB>();
  bar();
  x.from(ra, rb);
  x.read(0);
  ready_b(2);
  for (int kt = 0; kt < p.nk; ++kt) {
    // here: A's stage kt + 1 has gone out, of B's stage kt + 2 nothing yet
    substep(0, b_low);
    substep(1, b_high);
    wb = next_b(wb);
    wa = ra;
    ra = next_a(ra);
    rb = next_b(rb);
    ready_a(kt + 2);
    substep(2, [](auto) {});
    x.from(ra, rb);
    settle<NB>();
    bar();  // stage kt + 1 has landed, stage kt's buffers are free
    substep(3, a_both);
    ready_b(kt + 3);
  }
  vm_wait<0>();
  bar();  // no wave reads the stages any more, no copy is under way
  epilogue<E, W, EPI, SPLIT>(g, p, wm, wn, lane, reinterpret_cast<float*>(smem) + wave * 32 * W::PITCH, x.acc);
}

// 256 x 128 tile, four waves of 128 x 64, three buffers of kBK, one workgroup per CU:
// a quarter less LDS traffic per product than 128 x 128, in half the pieces of 256 x
// 256, for products whose tiles make one even round.  Work is spread as there: after
// a substep's eight products come a fragment of the next substep and, every second
// time in three of the four substeps, a copy of the stage that goes where stage kt
// was (three copies in all four take as long, six in two of them 5 % longer).  1024 x
// 7168 x 4096: 51.9 us, 128 x 128 57.8, 256 x 256 75.4; 4096 x 1408 x 4096 45.7, 48.9, 73.5.
template <class E, bool ACOL, bool BCOL, int EPI, bool SPLIT>
__global__ __launch_bounds__(256, 1) void dense_gemm_wide_kernel(DenseGemm g, int tiles_m, int tiles_n, int splits) {
  constexpr int BM = 256, BN = 128;
  using W = Waves<BM, BN, 2, 2, EPI>;
  using A = Operand<BM, ACOL, 4, 1>;
  using B = Operand<BN, BCOL, 4, W::DUAL ? 2 : 1>;
  constexpr int STAGES = 3, STAGE = A::kBytes + B::kBytes, N_DMA = 12;
  static_assert(A::kCopies + B::kCopies == N_DMA && W::TM * W::TN == 8 && W::kEpilogueBytes <= STAGES * STAGE, "four copies in three substeps");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[STAGES * STAGE];

  Place p;
  if (!place_of<BM, W::NC>(g, tiles_m, tiles_n, splits, p)) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / 2, wn = wave % 2;
  A a;
  B b;
  a.start(g.a, p.m0, g.M, g.K, p.k_first, 0);
  b.start(g.b, p.n0, g.N, g.K, p.k_first, g.N);
  a.offsets(wave, lane);
  b.offsets(wave, lane);
  auto ready = [&](int kt) {
    a.step(p.k_first + kt * kBK, p.k_end);
    b.step(p.k_first + kt * kBK, p.k_end);
  };
  const uint32_t smem0 = lds_addr(smem), mine = wave * 1024;
  auto copy = [&](auto i, uint32_t buf) {
    if constexpr (i < A::kCopies) a.template copy<i>(buf + mine);
    else b.template copy<i - A::kCopies>(buf + A::kBytes + mine);
  };
  uint32_t rd = smem0, wr = smem0;  // the buffers of stage kt and of the stage being copied
  auto next = [&](uint32_t at) { return at + STAGE == smem0 + STAGES * STAGE ? smem0 : at + STAGE; };
  Math<E, W, A, B> x;
  x.start(wm * W::WTM, W::bfirst(wn), lane);
  // substep kk, the next one's six fragments, and copies FROM .. FROM + 3 (none from N_DMA on)
  auto substep = [&](int kk, auto from) {
    x.multiply(kk, [&](auto n) {
      if constexpr (n < x.R) x.read((kk + 1) % 4, n);
      if constexpr (n % 2 == 1 && from < N_DMA) copy(std::integral_constant<int, from + n / 2>{}, wr);
    });
  };

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    ready(s);
    each<N_DMA>([&](auto i) { copy(i, wr); });
    wr = next(wr);
  }
  ready(STAGES - 1);
  each<4>([&](auto i) { copy(i, wr); });
  vm_wait<N_DMA + 4>();
  bar();
  x.from(rd, rd + A::kBytes);
  x.read(0);
  for (int kt = 0; kt < p.nk; ++kt) {
    substep(0, std::integral_constant<int, 4>{});
    substep(1, std::integral_constant<int, 8>{});
    substep(2, std::integral_constant<int, N_DMA>{});
    ready(kt + STAGES);
    wr = rd;
    rd = next(rd);
    x.from(rd, rd + A::kBytes);
    settle<N_DMA>();
    bar();  // stage kt + 1 has landed, stage kt's buffer is free
    substep(3, std::integral_constant<int, 0>{});
  }
  vm_wait<0>();
  bar();  // no wave reads the stages any more, no copy is under way
  epilogue<E, W, EPI, SPLIT>(g, p, wm, wn, lane, reinterpret_cast<float*>(smem) + wave * 32 * W::PITCH, x.acc);
}

// The partial products of a split K, added in the order of the splits, and the epilogue.
template <class E, int EPI>
__global__ __launch_bounds__(64) void dense_join_kernel(DenseGemm g, int splits) {
  constexpr bool DUAL = EPI == kGlu;
  const size_t per_row = g.N / 8, n8 = static_cast<size_t>(g.M) * per_row;
  const int w = DUAL ? 2 * g.N : g.N;
  for (size_t i = blockIdx.x * 64ul + threadIdx.x; i < n8; i += gridDim.x * 64ul) {
    const int m = static_cast<int>(i / per_row), n = static_cast<int>(i % per_row) * 8;
    Beside<E, EPI> x;
    x.load(g, m, n);
    // four splits' loads in flight at a time, added in the order of the splits
    f32x8 c{}, up{};
    const size_t part = static_cast<size_t>(g.M) * w;
    const float* p = g.part + static_cast<size_t>(m) * w + n;
    for (int s = 0; s < splits; s += 4, p += 4 * part) {
      f32x8 v[4], u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float* at = p + (s + q < splits ? q : 0) * part;
        v[q] = load8<float>(at);
        if (DUAL) u[q] = load8<float>(at + g.N);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (s + q < splits) {
          c += v[q];
          if (DUAL) up += u[q];
        }
    }
    finish8<E, EPI>(g, m, n, c, up, x);
  }
}

namespace {

// Which tile, and in how many parts of K.
enum Tile { kSmall, k64, k128, k128Deep, k256x128, k256 };
struct Plan {
  Tile tile;
  int splits;
};
struct TileCost {
  int rows, cols, slots;  // tile, and how many run at once on the chip (256 CUs)
  // us: launch, first loads and epilogue; a step with one, two and more per CU
  float start, one, two, more;
};
// 64 x 64 and 64 x 128 (three buffers) and 128 x 128 (two) run three, two and two to a
// CU, 128 x 128 with three buffers, 256 x 128 and 256 x 256 one.  Fitted to 1900 timings
// of 104 products, of 20 to 8000 rows, and for 256 x 128 of 57: what the figures choose
// takes 1 % more than the quickest on average (3 % more without 256 x 128).  Among them,
// us, on the six in this order: 512 x 2048 x 1408 7.6, 9.2, 12.2, 11.9, 17.4, 30.9; 777 x
// 4096 x 2816 38, 29, 31, 23, 31, 53; 2048 x 4096 x 2816 74, 59, 46, 49, 42, 59; 2816 x 4096
// x 2048 73, 62, 55, 54, 54, 48.  They know neither the bytes of an epilogue nor that the
// clock falls in long runs: 8192 x 4096 x 11264, 404 us by them, takes 550, and with kDglu's
// 1.3 GB (8192 x 11264 x 4096) 840 for 486.
constexpr TileCost kTiles[] = {
    {64, 64, 768, 3.5f, 0.20f, 0.44f, 0.63f},
    {64, 128, 512, 3.5f, 0.29f, 0.76f, 0.76f},
    {128, 128, 512, 4.8f, 0.48f, 0.87f, 0.87f},
    {128, 128, 256, 4.1f, 0.44f, 0.44f, 0.44f},
    {256, 128, 256, 5.6f, 0.70f, 0.70f, 0.70f},
    {256, 256, 256, 11.9f, 1.08f, 1.08f, 1.08f},
};
// The time that a product takes by those figures: rounds of tiles, and where K is
// split the launch that joins the parts and their traffic.  128 x 2048 (gate and up)
// x 7168: 33 us whole and 19.6 in three parts; 512 x 2048 x 1408 (64 x 128
// tiles): 8.9 whole, 12.4 in two.
float cost_of(const TileCost& t, bool dual, int M, int N, int K, int splits) {
  const int cols = dual ? t.cols / 2 : t.cols;
  const long tiles = static_cast<long>((M + t.rows - 1) / t.rows) * ((N + cols - 1) / cols) * splits;
  const int steps = ((K + kBK - 1) / kBK + splits - 1) / splits;
  const long rest = tiles % t.slots;
  float us = static_cast<float>(tiles / t.slots) * (t.start + t.more * steps);
  if (rest) us += t.start + (rest <= 256 ? t.one : rest <= 512 ? t.two : t.more) * steps;
  if (splits > 1) us += 1.2f + 0.22f * splits + (splits + 1) * 4e-6f * M * N * (dual ? 2 : 1) / 3.2f;
  return us;
}

// K is split into one of these numbers of parts, of two steps or more, while the
// partial products stay below 2^25 elements.
constexpr int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16};
constexpr long kMostPart = 1L << 25;

Plan plan_for(int epi, int M, int N, int K) {
  const bool dual = epi == kGlu;
  const int nk = (K + kBK - 1) / kBK;
  Plan best{k64, 1};
  float least = 0.f;
  for (int t = dual ? k64 : kSmall; t <= k256; ++t)  // the smallest has no gate and up pairs
    for (int splits : kSplits) {
      if (splits > 1 && (nk < 2 * splits || splits * static_cast<long>(M) * N * (dual ? 2 : 1) > kMostPart)) break;
      const float us = cost_of(kTiles[t], dual, M, N, K, splits);
      if (least == 0.f || us < least) {
        least = us;
        best = {static_cast<Tile>(t), splits};
      }
    }
  return best;
}

// Launches a tile kernel, the whole of K or one of its splits per workgroup, and
// what joins the splits.
template <class E, int BM, int BN, int EPI, class K>
hipError_t run_tile(const DenseGemm& g, int splits, K whole, K part, hipStream_t s) {
  constexpr int NC = EPI == kGlu ? BN / 2 : BN;
  const int tm = (g.M + BM - 1) / BM, tn = (g.N + NC - 1) / NC;
  const long total = static_cast<long>(tm) * tn * splits;
  const dim3 grid(static_cast<unsigned>((total + 7) / 8 * 8)), block(256);
  const K kernel = splits == 1 ? whole : part;
  kernel<<<grid, block, 0, s>>>(g, tm, tn, splits);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const size_t n8 = static_cast<size_t>(g.M) * (g.N / 8);
  dense_join_kernel<E, EPI><<<static_cast<unsigned>(std::min<size_t>((n8 + 63) / 64, 8192)), 64, 0, s>>>(g, splits);
  return hipGetLastError();
}

template <class E, bool ACOL, bool BCOL, int EPI>
hipError_t run(const DenseGemm& g, hipStream_t s) {
  const Plan p = plan_for(EPI, g.M, g.N, g.K);
  if constexpr (EPI != kGlu) {
    if (p.tile == kSmall)
      return run_tile<E, 64, 64, EPI>(g, p.splits, dense_gemm_64_kernel<E, 64, ACOL, BCOL, EPI, false>,
                                      dense_gemm_64_kernel<E, 64, ACOL, BCOL, EPI, true>, s);
  }
  switch (p.tile) {
    case k64:
      return run_tile<E, 64, 128, EPI>(g, p.splits, dense_gemm_64_kernel<E, 128, ACOL, BCOL, EPI, false>,
                                       dense_gemm_64_kernel<E, 128, ACOL, BCOL, EPI, true>, s);
    case k128:
      return run_tile<E, 128, 128, EPI>(g, p.splits, dense_gemm_128_kernel<E, 2, ACOL, BCOL, EPI, false>,
                                        dense_gemm_128_kernel<E, 2, ACOL, BCOL, EPI, true>, s);
    case k128Deep:
      return run_tile<E, 128, 128, EPI>(g, p.splits, dense_gemm_128_kernel<E, 3, ACOL, BCOL, EPI, false>,
                                        dense_gemm_128_kernel<E, 3, ACOL, BCOL, EPI, true>, s);
    case k256x128:
      return run_tile<E, 256, 128, EPI>(g, p.splits, dense_gemm_wide_kernel<E, ACOL, BCOL, EPI, false>,
                                        dense_gemm_wide_kernel<E, ACOL, BCOL, EPI, true>, s);
    default:
      return run_tile<E, 256, 256, EPI>(g, p.splits, dense_gemm_256_kernel<E, ACOL, BCOL, EPI, false>,
                                        dense_gemm_256_kernel<E, ACOL, BCOL, EPI, true>, s);
  }
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

// What the plan for any number of the block's rows up to these may ask for, not what
// the plan for these does: fewer rows are often split more (256 rows of 7168 x 2048
// take 17 MB of partial products, 512 none), and a caller sizes for its largest batch.
size_t dense_gemm_workspace_bytes(int layout, int epi, int M, int N, int K) {
  if (dense_rows_fits(layout, epi, M, N, K)) return 0;
  const int nk = (K + kBK - 1) / kBK;
  const long whole = static_cast<long>(M) * N * (epi == kGlu ? 2 : 1);
  long most = 0;
  for (int splits : kSplits) {
    if (splits == 1 || nk < 2 * splits) continue;
    if (layout != kColCol) most = std::min(splits * whole, kMostPart);  // M of them or fewer
    else if (splits * whole <= kMostPart) most = splits * whole;        // a sum over K of them or fewer
  }
  return static_cast<size_t>(most) * 4;
}

hipError_t launch_dense_gemm(int dtype, int layout, int epi, const DenseGemm& g, hipStream_t s) {
  if (dense_rows_fits(layout, epi, g.M, g.N, g.K)) return launch_dense_rows(dtype, epi, g, s);
  return dtype == kBf16 ? run_type<bf16_t>(layout, epi, g, s) : run_type<f16_t>(layout, epi, g, s);
}

}  // namespace moe
