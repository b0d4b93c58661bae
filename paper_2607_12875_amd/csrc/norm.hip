// Layer and rms norm over the rows of x [T, H], forward and backward: the norm in
// front of the router or of a feed-forward block.
//   s = round(x + residual);  xhat = (s - mean) rstd  (rms: s rstd)
//   y = xhat w + b
//   g = dy w;  dx = rstd (g - mean(g) - xhat mean(g xhat)) + dsum  (rms: no mean(g))
//   dw = sum over rows of dy xhat;  db = sum over rows of dy
// All of it is bound by HBM, so a row is read once and held in registers: a row
// group of G threads, each with NV chunks of 16 bytes.  The variance is summed
// about the mean, in a second pass over the registers.  A width that no chunk
// divides leaves rows off their 16-byte alignment, which the memory takes, and a
// last chunk that is read element by element.
#include <algorithm>

#include "common.hpp"
#include "dense.hpp"
#include "dense_math.hpp"

namespace moe {

namespace {

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

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Sums of N values over the G threads of a row group (G a power of two, at least a
// wave); `slots` holds N floats per wave of the workgroup.  Groups of several waves
// meet in LDS, added in wave order, so every thread has the same sums.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int G, float* slots) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if (G == kWave) return;
  const int wave = threadIdx.x / kWave, nw = G / kWave, first = wave / nw * nw;
  if (lane_id() == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) slots[wave * N + i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.f;
    for (int w = 0; w < nw; ++w) v[i] += slots[(first + w) * N + i];
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

// Each workgroup takes every gridDim-th set of rows, its row groups one each, and
// keeps its columns' sums of dy xhat and dy in registers; at the end the groups'
// sums are joined in LDS, in order, and written as one row of partial sums.
template <class E, int NV, int KIND>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormBackward a, int G) {
  using C = Chunk<E>;
  __shared__ float slots[2][2 * 16];
  extern __shared__ float joined[];  // [2][H] with more than one row group
  const int groups = blockDim.x / G, gi = threadIdx.x / G, gt = threadIdx.x % G;
  float dw[NV][C::W], db[NV][C::W], w[NV][C::W];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    C::load(static_cast<const E*>(a.weight), gt + i * G, a.H, w[i]);
#pragma unroll
    for (int e = 0; e < C::W; ++e) dw[i][e] = db[i][e] = 0.f;
  }
  const float inv = 1.0f / a.H;
  int turn = 0;
  for (int r0 = blockIdx.x * groups; r0 < a.T; r0 += gridDim.x * groups, turn ^= 1) {
    const int row = r0 + gi;
    const bool live = row < a.T;
    const size_t at = static_cast<size_t>(live ? row : r0) * a.H;
    float x[NV][C::W], g[NV][C::W];
    const float rstd = a.rstd[live ? row : r0], mean = KIND == kLayerNorm ? a.mean[live ? row : r0] : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      C::load(static_cast<const E*>(a.x) + at, gt + i * G, a.H, x[i]);
      C::load(static_cast<const E*>(a.dy) + at, gt + i * G, a.H, g[i]);
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < C::W; ++e) {
        x[i][e] = (x[i][e] - mean) * rstd;
        if (live) {
          dw[i][e] = fmaf(g[i][e], x[i][e], dw[i][e]);
          db[i][e] += g[i][e];
        }
        g[i][e] *= w[i][e];
        sum[0] += g[i][e];
        sum[1] = fmaf(g[i][e], x[i][e], sum[1]);
      }
    group_sum(sum, G, slots[turn]);
    if (!live) continue;
    const float s1 = KIND == kLayerNorm ? sum[0] * inv : 0.f, s2 = sum[1] * inv;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = gt + i * G;
      if (c * C::W >= a.H) continue;
      float d[C::W] = {};
      if (a.dsum) C::load(static_cast<const E*>(a.dsum) + at, c, a.H, d);
#pragma unroll
      for (int e = 0; e < C::W; ++e) d[e] = fmaf(rstd, g[i][e] - s1 - x[i][e] * s2, d[e]);
      C::store(static_cast<E*>(a.dx) + at, c, a.H, d);
    }
  }
  if (!a.part) return;
  for (int q = groups - 1; q > 0; --q) {  // group 0 ends with the sums of all
    if (gi == q) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < C::W; ++e) {
          const int h = (gt + i * G) * C::W + e;
          if (h < a.H) {
            if (q < groups - 1) {
              joined[h] += dw[i][e];
              joined[a.H + h] += db[i][e];
            } else {
              joined[h] = dw[i][e];
              joined[a.H + h] = db[i][e];
            }
          }
        }
    }
    __syncthreads();
  }
  if (gi) return;
  float* part = a.part + static_cast<size_t>(blockIdx.x) * 2 * a.H;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < C::W; ++e) {
      const int h = (gt + i * G) * C::W + e;
      if (h < a.H) {
        part[h] = dw[i][e] + (groups > 1 ? joined[h] : 0.f);
        part[a.H + h] = db[i][e] + (groups > 1 ? joined[a.H + h] : 0.f);
      }
    }
}

// Column sums of the partial rows: 64 columns per workgroup, sixteen slices of the rows.
__global__ __launch_bounds__(1024) void norm_columns_kernel(const float* part, int rows, int H, float* dweight, float* dbias) {
  __shared__ float s[16][kWave];
  float* out = blockIdx.y ? dbias : dweight;
  if (!out) return;
  const int l = threadIdx.x % kWave, q = threadIdx.x / kWave, h = blockIdx.x * kWave + l;
  float v = 0.f;
  if (h < H)
    for (int r = q; r < rows; r += 16) v += part[(static_cast<size_t>(r) * 2 + blockIdx.y) * H + h];
  s[q][l] = v;
  __syncthreads();
  if (q == 0 && h < H) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += s[i][l];
    out[h] = v;
  }
}

// Threads per row and chunks per thread: H / W chunks over a power of two of
// threads.
struct Shape {
  int G, NV;
};
Shape shape_of(int H, int width, int most) {
  const int chunks = (H + width - 1) / width;
  Shape s{kWave, 1};
  while (s.G < 1024 && s.G * most < chunks) s.G *= 2;
  while (s.G * s.NV < chunks) s.NV *= 2;
  return s;
}

int backward_threads(const Shape& s) { return std::max(s.G, 512); }
int backward_blocks(int T, int groups) { return std::min(kNormBlocks, (T + groups - 1) / groups); }

template <class E, int KIND, class F>
hipError_t with_nv(int nv, F f) {
  switch (nv) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

template <class E, int KIND>
hipError_t forward(const NormForward& a, hipStream_t s) {
  const Shape p = shape_of(a.H, Chunk<E>::W, a.T >= 1024 ? 4 : 1);
  const int threads = std::max(256, p.G), rows = threads / p.G;
  return with_nv<E, KIND>(p.NV, [&](auto nv) {
    norm_forward_kernel<E, decltype(nv)::value, KIND><<<(a.T + rows - 1) / rows, threads, 0, s>>>(a, p.G);
    return hipGetLastError();
  });
}

template <class E, int KIND>
hipError_t backward(const NormBackward& a, hipStream_t s) {
  const Shape p = shape_of(a.H, Chunk<E>::W, 2);
  const int threads = backward_threads(p), groups = threads / p.G, blocks = backward_blocks(a.T, groups);
  const size_t lds = groups > 1 ? 2ul * a.H * 4 : 0;
  if (a.T > 0) {
    const hipError_t e = with_nv<E, KIND>(p.NV, [&](auto nv) {
      norm_backward_kernel<E, decltype(nv)::value, KIND><<<blocks, threads, lds, s>>>(a, p.G);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  norm_columns_kernel<<<dim3((a.H + kWave - 1) / kWave, 2), 1024, 0, s>>>(a.part, blocks, a.H, a.dweight, a.dbias);
  return hipGetLastError();
}

}  // namespace

size_t norm_backward_workspace_bytes(int T, int H) {
  return static_cast<size_t>(std::min(kNormBlocks, T)) * 2 * H * 4;
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
