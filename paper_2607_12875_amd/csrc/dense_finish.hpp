// The epilogues of the feed-forward block's products, on eight columns of one row.
// All of it is fp32 until the store.  h and dpre are rounded to the type there, since
// the products that read them take 16-bit operands; the same rounding in a plain form
// in fp32 gives these results to 1.3e-4 .. 2.4e-4 (2-norm, bf16; the rest is sums in
// another order that round to the other side), without it they differ by 1.7e-3 ..
// 2.6e-3 (fp16 3.2e-4).  pre, which only this epilogue reads again, stays fp32.
#pragma once
#include "dense.hpp"
#include "dense_math.hpp"

namespace moe {

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

}  // namespace moe
