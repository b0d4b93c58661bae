// Layer and rms norm over the rows of x [T, H], forward and backward: the norm in
// front of the router or of a feed-forward block.
//   s = round(x + residual);  xhat = (s - mean) rstd  (rms: s rstd)
//   y = xhat w + b
//   g = dy w;  dx = rstd (g - mean(g) - xhat mean(g xhat)) + dsum  (rms: no mean(g))
//   dw = sum over rows of dy xhat;  db = sum over rows of dy
// All of it is bound by HBM, so a row is read once and held in registers: a row
// group of G threads, whole waves, each with NV chunks of 16 bytes.  Narrow rows leave
// lanes of their wave idle: 262144 x 128 bf16, 16 of 64, runs at 2.0 TB/s forward.
// The variance is summed about the mean, in a second pass over the registers.  A
// width that no chunk divides leaves rows off their 16-byte alignment, which the
// memory takes, and a last chunk that is read element by element.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "dense.hpp"
#include "dense_math.hpp"

namespace moe {

namespace {

constexpr int kLaunchRows = 1 << 21;  // of the forward pass
constexpr int kMostLds = 158 * 1024;  // column sums in LDS, beside 256 bytes of its own
constexpr int kNormBlocks = 256;  // workgroups of the backward pass at most: one per CU

template <class E> struct Chunk {
  static constexpr int W = 16 / sizeof(E);
  struct __attribute__((packed, aligned(sizeof(E)))) Bits { u32x4 v; };
  // elements [c W, c W + W) of a row of H; those past H are zero
  __device__ static void load(const E* row, int c, int H, float (&f)[W]) {
    if (c * W + W <= H) {
      const u32x4 b = reinterpret_cast<const Bits*>(row + c * W)->v;
      unpack(b, f);
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e) f[e] = c * W + e < H ? static_cast<float>(row[c * W + e]) : 0.f;
    }
  }
  __device__ static u32x4 raw(const E* row, int c, int H) {
    if (c * W + W <= H) return reinterpret_cast<const Bits*>(row + c * W)->v;
    typedef E V __attribute__((ext_vector_type(W)));
    V v;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = c * W + e < H ? row[c * W + e] : static_cast<E>(0.f);
    return __builtin_bit_cast(u32x4, v);
  }
  __device__ static void store(E* row, int c, int H, const float (&f)[W]) {
    if (c * W + W <= H) {
      reinterpret_cast<Bits*>(row + c * W)->v = pack(f);
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (c * W + e < H) row[c * W + e] = static_cast<E>(f[e]);
    }
  }
  __device__ static void unpack(const u32x4& b, float (&f)[W]) {
    typedef E V __attribute__((ext_vector_type(W)));
    const V v = __builtin_bit_cast(V, b);
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = static_cast<float>(v[e]);
  }
  __device__ static u32x4 pack(const float (&f)[W]) {
    typedef E V __attribute__((ext_vector_type(W)));
    V v;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = static_cast<E>(f[e]);
    return __builtin_bit_cast(u32x4, v);
  }
};

// Sum over the wave: four DPP permutes inside each row of sixteen lanes, then the
// four rows' sums as scalars.
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = dpp_add<0xB1>(v);   // quad_perm 1 0 3 2
  v = dpp_add<0x4E>(v);   // quad_perm 2 3 0 1
  v = dpp_add<0x141>(v);  // row_half_mirror
  v = dpp_add<0x140>(v);  // row_mirror
  auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// Sums of N values over the G threads of a row group (one to sixteen waves);
// `slots` holds N floats per wave of the workgroup.  Groups of several waves meet in
// LDS: a lane per wave reads its sum, and the row of sixteen lanes adds them.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int G, float* slots) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if (G == kWave) return;
  const int wave = threadIdx.x / kWave, nw = G / kWave, first = wave / nw * nw, l = lane_id() & 15;
  if (lane_id() == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) slots[wave * N + i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float s = l < nw ? slots[(first + l) * N + i] : 0.f;
    v[i] = dpp_add<0x140>(dpp_add<0x141>(dpp_add<0x4E>(dpp_add<0xB1>(s))));
  }
}

template <class E, int NV, int KIND>
__global__ __launch_bounds__(1024) void norm_forward_kernel(NormForward a, int G) {
  using C = Chunk<E>;
  __shared__ float slots[2][16];
  const int gi = threadIdx.x / G, gt = threadIdx.x % G;
  const int row = blockIdx.x * (blockDim.x / G) + gi;
  const bool live = row < a.T;
  const size_t at = static_cast<size_t>(live ? row : 0) * a.H;
  float s[NV][C::W];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = gt + i * G;
    C::load(static_cast<const E*>(a.x) + at, c, a.H, s[i]);
  }
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = gt + i * G;
      float r[C::W];
      C::load(static_cast<const E*>(a.residual) + at, c, a.H, r);
#pragma unroll
      for (int e = 0; e < C::W; ++e) s[i][e] += r[e];
      if constexpr (C::W > 4) C::unpack(C::pack(s[i]), s[i]);
      if (live && c * C::W < a.H) C::store(static_cast<E*>(a.sum) + at, c, a.H, s[i]);
    }
  }
  float mean = 0.f, sum[1];
  if constexpr (KIND == kLayerNorm) {
    sum[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < C::W; ++e) sum[0] += s[i][e];
    group_sum(sum, G, slots[0]);
    mean = sum[0] / a.H;
  }
  sum[0] = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < C::W; ++e) {
      if (KIND == kLayerNorm) s[i][e] = (gt + i * G) * C::W + e < a.H ? s[i][e] - mean : 0.f;
      sum[0] = fmaf(s[i][e], s[i][e], sum[0]);
    }
  group_sum(sum, G, slots[1]);
  const float rstd = 1.0f / sqrtf(sum[0] / a.H + a.eps);
  if (!live) return;
  if (gt == 0) {
    if (KIND == kLayerNorm && a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = gt + i * G;
    if (c * C::W >= a.H) continue;
    float w[C::W], b[C::W] = {};
    C::load(static_cast<const E*>(a.weight), c, a.H, w);
    if (a.bias) C::load(static_cast<const E*>(a.bias), c, a.H, b);
#pragma unroll
    for (int e = 0; e < C::W; ++e) w[e] = fmaf(s[i][e] * rstd, w[e], b[e]);
    C::store(static_cast<E*>(a.y) + at, c, a.H, w);
  }
}

// Four columns of a row of sums from column h on (16-byte aligned), up to `end`.
__device__ __forceinline__ void put4(float* row, int h, int end, const f32x4& v) {
  if (!row) return;
  if (h + 4 <= end) {
    *reinterpret_cast<f32x4*>(row + h) = v;
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (h + q < end) row[h + q] = v[q];
  }
}

// Each workgroup takes every gridDim-th set of rows, its row groups one each, and
// keeps its columns' sums of dy xhat and dy in registers; at the end the groups'
// sums are joined in LDS, in order, and written as one row of partial sums.  The
// next rows are in flight, unconverted, while a row is reduced and written: without,
// the barrier of every row stood between the loads (8192 x 4096 bf16 with dsum, 268
// MB: 102 us; 46 now).  Rows so wide that a thread has several chunks keep
// the column sums in LDS (IN_LDS; each thread its own columns, so without atomics),
// where they fit, to 20224 elements.  With two chunks all else stays in registers
// (2048 x 16384 bf16, 201 MB: 44 us).  With more, 16-bit rows past 16384 elements and
// fp32 rows past 8192, the 128 registers of 1024 threads do not hold the row, the
// next one and the weight, nor the sums past LDS: four fp32 chunks spill 110 bytes a
// lane (4096 x 16384, 805 MB: 184 us), four 16-bit ones 0.5 to 0.7 KB (4096 x 18432 bf16, 453
// MB: 300 us), eight 0.7 to 1.8 KB (1024 x 40008 bf16, 246 MB: 735 us), sixteen 2 KB.
template <class E, int NV, int KIND, bool IN_LDS>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormBackward a, int G) {
  using C = Chunk<E>;
  constexpr int W = C::W, NR = IN_LDS ? 1 : NV;
  __shared__ float slots[2][2 * 16];
  extern __shared__ __attribute__((aligned(16))) float joined[];  // IN_LDS: [2][H up to whole chunks], the sums; else the row groups' sums at the end
  const int groups = blockDim.x / G, gi = threadIdx.x / G, gt = threadIdx.x % G, Hp = (a.H + 7) / 8 * 8;
  float dw[NR][W], db[NR][W];
  u32x4 w[NV], x1[NV], g1[NV], d1[NV];  // weight; the next row's x, dy, dsum
  float mean1 = 0.f, rstd1 = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w[i] = C::raw(static_cast<const E*>(a.weight), gt + i * G, a.H);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const int h = (gt + i * G) * W + e;
      if constexpr (!IN_LDS) dw[i][e] = db[i][e] = 0.f;
      else if (h < Hp) joined[h] = joined[Hp + h] = 0.f;
    }
  }
  auto fetch = [&](int r0) {
    const int row = min(r0 + gi, a.T - 1);
    const size_t at = static_cast<size_t>(row) * a.H;
    rstd1 = a.rstd[row];
    if (KIND == kLayerNorm) mean1 = a.mean[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x1[i] = C::raw(static_cast<const E*>(a.x) + at, gt + i * G, a.H);
      g1[i] = C::raw(static_cast<const E*>(a.dy) + at, gt + i * G, a.H);
    }
  };
  auto fetch_dsum = [&](int r0) {
    const size_t at = static_cast<size_t>(min(r0 + gi, a.T - 1)) * a.H;
#pragma unroll
    for (int i = 0; i < NV; ++i) d1[i] = C::raw(static_cast<const E*>(a.dsum) + at, gt + i * G, a.H);
  };
  const float inv = 1.0f / a.H;
  const int stride = gridDim.x * groups;
  int turn = 0;
  fetch(blockIdx.x * groups);
  if (a.dsum) fetch_dsum(blockIdx.x * groups);
  for (int r0 = blockIdx.x * groups; r0 < a.T; r0 += stride, turn ^= 1) {
    const bool live = r0 + gi < a.T;
    const size_t at = static_cast<size_t>(r0 + gi) * a.H;
    const float rstd = rstd1, mean = mean1;
    float x[NV][W], g[NV][W];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      C::unpack(x1[i], x[i]);
      C::unpack(g1[i], g[i]);
    }
    if (r0 + stride < a.T) fetch(r0 + stride);
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float wf[W];
      C::unpack(w[i], wf);
      float* const sw = joined + (gt + i * G) * W;
      const bool mine = (gt + i * G) * W < a.H;
#pragma unroll
      for (int e = 0; e < W; ++e)  // past the row an exact zero: -mean * rstd may be past fp32
        x[i][e] = KIND != kLayerNorm || (gt + i * G) * W + e < a.H ? (x[i][e] - mean) * rstd : 0.f;
      if constexpr (IN_LDS) {
        if (mine) {
#pragma unroll
          for (int e = 0; e < W; e += 4) {
            f32x4 vw = *reinterpret_cast<f32x4*>(sw + e), vb = *reinterpret_cast<f32x4*>(sw + Hp + e);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              vw[q] = fmaf(g[i][e + q], x[i][e + q], vw[q]);
              vb[q] += g[i][e + q];
            }
            *reinterpret_cast<f32x4*>(sw + e) = vw;
            *reinterpret_cast<f32x4*>(sw + Hp + e) = vb;
          }
        }
      } else if (live) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          dw[i][e] = fmaf(g[i][e], x[i][e], dw[i][e]);
          db[i][e] += g[i][e];
        }
      }
#pragma unroll
      for (int e = 0; e < W; ++e) {
        g[i][e] *= wf[e];
        sum[0] += g[i][e];
        sum[1] = fmaf(g[i][e], x[i][e], sum[1]);
      }
    }
    group_sum(sum, G, slots[turn]);
    if (live) {
      const float s1 = KIND == kLayerNorm ? sum[0] * inv : 0.f, s2 = sum[1] * inv;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = gt + i * G;
        if (c * W >= a.H) continue;
        float d[W] = {};
        if (a.dsum) C::unpack(d1[i], d);
#pragma unroll
        for (int e = 0; e < W; ++e) d[e] = fmaf(rstd, g[i][e] - s1 - x[i][e] * s2, d[e]);
        C::store(static_cast<E*>(a.dx) + at, c, a.H, d);
      }
    }
    if (a.dsum && r0 + stride < a.T) fetch_dsum(r0 + stride);
  }
  if (!a.dweight && !a.dbias) return;
  // with one workgroup its sums are the results, else a row of partial sums
  float* const pw = gridDim.x == 1 ? a.dweight : a.part + static_cast<size_t>(blockIdx.x) * 2 * Hp;
  float* const pb = gridDim.x == 1 ? a.dbias : pw + Hp;
  if (!IN_LDS && groups > 1) {  // [group][2][G W]: every group's sums meet, in the order of the groups
    const int width = G * W;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      joined[gi * 2 * width + gt * W + e] = dw[0][e];
      joined[(gi * 2 + 1) * width + gt * W + e] = db[0][e];
    }
    __syncthreads();
    for (int h = threadIdx.x; h < a.H; h += blockDim.x) {
      float sw = joined[h], sb = joined[width + h];
      for (int q = 1; q < groups; ++q) {
        sw += joined[q * 2 * width + h];
        sb += joined[(q * 2 + 1) * width + h];
      }
      if (pw) pw[h] = sw;
      if (pb) pb[h] = sb;
    }
    return;
  }
  const int end = gridDim.x == 1 ? a.H : Hp;  // partial rows are whole chunks
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int h = (gt + i * G) * W;
    if (h >= a.H) continue;
#pragma unroll
    for (int e = 0; e < W; e += 4) {
      f32x4 vw, vb;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        vw[q] = IN_LDS ? joined[h + e + q] : dw[IN_LDS ? 0 : i][e + q];
        vb[q] = IN_LDS ? joined[Hp + h + e + q] : db[IN_LDS ? 0 : i][e + q];
      }
      put4(pw, h + e, end, vw);
      put4(pb, h + e, end, vb);
    }
  }
}

// Column sums of the partial rows: 64 columns per workgroup, four per thread, 64
// slices of the rows.
__global__ __launch_bounds__(1024) void norm_columns_kernel(const float* part, int rows, int H, float* dweight, float* dbias) {
  __shared__ f32x4 s[64][16];
  float* out = blockIdx.y ? dbias : dweight;
  if (!out) return;
  const int l = threadIdx.x % 16, q = threadIdx.x / 16, h = (blockIdx.x * 16 + l) * 4, Hp = (H + 7) / 8 * 8;
  f32x4 v{};
  if (h < H)
#pragma unroll 4
    for (int r = q; r < rows; r += 64) v += *reinterpret_cast<const f32x4*>(part + (static_cast<size_t>(r) * 2 + blockIdx.y) * Hp + h);
  s[q][l] = v;
  __syncthreads();
  if (q >= 4) return;
  // four waves' worth of column groups: 16 slices each, then the four
  for (int i = 1; i < 16; ++i) v += s[q + 4 * i][l];
  s[q][l] = v;
  __atomic_signal_fence(__ATOMIC_SEQ_CST);  // one wave: its reads follow its writes
  __builtin_amdgcn_wave_barrier();
  if (q == 0 && h < H) {
    v = (v + s[1][l]) + (s[2][l] + s[3][l]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (h + e < H) out[h + e] = v[e];
  }
}

__global__ void norm_zero_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n && a) a[i] = 0.f;
  if (i < n && b) b[i] = 0.f;
}

// Threads per row (whole waves) and chunks per thread, at most `most` of them
// where 1024 threads can have the row.
struct Shape {
  int G, NV;
};
Shape shape_of(int H, int width, int most) {
  const int chunks = (H + width - 1) / width;
  Shape s{std::min(1024, ((chunks + most - 1) / most + kWave - 1) / kWave * kWave), 1};
  while (s.G * s.NV < chunks) s.NV *= 2;
  return s;
}

// Up to two rows per row group one workgroup does all, in one launch.
// Otherwise each takes the same number of rows, or one less.
// More workgroups than CUs write more partial sums than they save (777 x 5120: 14.3
// us, with two per CU 16.5).
int backward_blocks(int T, int groups) {
  if (T <= 2 * groups) return 1;
  const int sets = (T + groups - 1) / groups, each = (sets + kNormBlocks - 1) / kNormBlocks;
  return (sets + each - 1) / each;
}

// f with a thread's chunks as a constant; rows of more than 1024 W elements have
// several, up to kMostWidth.
template <class E, int NV = 1, class F> hipError_t with_nv(int nv, F f) {
  if constexpr (1024 * Chunk<E>::W * NV < kMostWidth) {
    if (nv > NV) return with_nv<E, 2 * NV>(nv, f);
  }
  return f(std::integral_constant<int, NV>{});
}

// Bytes of both column sums of a row.
constexpr int sums_bytes(int H) { return 2 * ((H + 7) / 8 * 8) * 4; }

template <class E, int KIND>
hipError_t forward(NormForward a, hipStream_t s) {
  // few rows: as many threads as a row can use; many: two chunks each (8192 x 7168
  // bf16 with residual 86 us, with four 92, 777 x 5120 7.2, with one 9.0)
  const Shape p = shape_of(a.H, Chunk<E>::W, a.T >= 512 ? 2 : 1);
  const int rows = std::max(1, 256 / p.G), threads = rows * p.G;
  // a launch has fewer than 2^32 threads
  for (int left = a.T; left > 0; left -= kLaunchRows) {
    a.T = std::min(left, kLaunchRows);
    const hipError_t e = with_nv<E>(p.NV, [&](auto nv) {
      norm_forward_kernel<E, decltype(nv)::value, KIND><<<(a.T + rows - 1) / rows, threads, 0, s>>>(a, p.G);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    const size_t n = static_cast<size_t>(a.T) * a.H;
    a.x = static_cast<const E*>(a.x) + n;
    a.y = static_cast<E*>(a.y) + n;
    if (a.residual) {
      a.residual = static_cast<const E*>(a.residual) + n;
      a.sum = static_cast<E*>(a.sum) + n;
    }
    if (a.mean) a.mean += a.T;
    if (a.rstd) a.rstd += a.T;
  }
  return hipSuccess;
}

template <class E, int KIND>
hipError_t backward(const NormBackward& a, hipStream_t s) {
  const Shape p = shape_of(a.H, Chunk<E>::W, 1);
  const int groups = p.NV > 1 ? 1 : 1024 / p.G, threads = groups * p.G, blocks = backward_blocks(a.T, groups);
  const int sums = sums_bytes(a.H);
  if (a.T > 0) {
    const hipError_t e = with_nv<E>(p.NV, [&](auto nv) {
      constexpr int NV = decltype(nv)::value, W = Chunk<E>::W;
      // the widths that take NV chunks: does a row's pair of sums fit the LDS?
      constexpr int least = 1024 * W * (NV / 2) + 1, most = std::min(1024 * W * NV, kMostWidth);
      constexpr bool never = NV == 1 || sums_bytes(least) > kMostLds, always = !never && sums_bytes(most) <= kMostLds;
      auto launch = [&](auto in_lds) {
        constexpr bool IN_LDS = decltype(in_lds)::value;
        if constexpr (IN_LDS) {
          const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(norm_backward_kernel<E, NV, KIND, true>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, kMostLds);
          if (e != hipSuccess) return e;
        }
        // several row groups have one chunk per thread each
        const int lds = IN_LDS ? sums : groups > 1 ? 2 * threads * W * 4 : 0;
        norm_backward_kernel<E, NV, KIND, IN_LDS><<<blocks, threads, lds, s>>>(a, p.G);
        return hipGetLastError();
      };
      if constexpr (never || always) return launch(std::bool_constant<always>{});
      else return sums <= kMostLds ? launch(std::true_type{}) : launch(std::false_type{});
    });
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  if (a.T == 0) norm_zero_kernel<<<(a.H + 255) / 256, 256, 0, s>>>(a.dweight, a.dbias, a.H);
  else if (blocks > 1) norm_columns_kernel<<<dim3((a.H + 63) / 64, 2), 1024, 0, s>>>(a.part, blocks, a.H, a.dweight, a.dbias);
  return hipGetLastError();
}

}  // namespace

size_t norm_backward_workspace_bytes(int T, int H) {
  return static_cast<size_t>(std::min(kNormBlocks, T)) * 2 * ((H + 7) / 8 * 8) * 4;
}

hipError_t launch_norm_forward(int dtype, int kind, const NormForward& a, hipStream_t s) {
  if (dtype == kF32) return kind == kLayerNorm ? forward<float, kLayerNorm>(a, s) : forward<float, kRmsNorm>(a, s);
  if (dtype == kBf16) return kind == kLayerNorm ? forward<bf16_t, kLayerNorm>(a, s) : forward<bf16_t, kRmsNorm>(a, s);
  return kind == kLayerNorm ? forward<f16_t, kLayerNorm>(a, s) : forward<f16_t, kRmsNorm>(a, s);
}

hipError_t launch_norm_backward(int dtype, int kind, const NormBackward& a, hipStream_t s) {
  if (dtype == kF32) return kind == kLayerNorm ? backward<float, kLayerNorm>(a, s) : backward<float, kRmsNorm>(a, s);
  if (dtype == kBf16) return kind == kLayerNorm ? backward<bf16_t, kLayerNorm>(a, s) : backward<bf16_t, kRmsNorm>(a, s);
  return kind == kLayerNorm ? backward<f16_t, kLayerNorm>(a, s) : backward<f16_t, kRmsNorm>(a, s);
}

}  // namespace moe
