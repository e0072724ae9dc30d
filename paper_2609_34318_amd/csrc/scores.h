// Device-side parts of the modified scores (hydra_scores.h): what a row sees, the cap, the bias.
//
// The kernels hold a 32 x 32 block of raw scores in the MFMA's result registers: element e of a lane is at
// offset 16 (e / 8) + e % 8 from the lane's first key (forward, dQ) or first query (dK/dV).  With a cap or
// slopes the scores are turned in place into log2 units, where the plain kernels fold the scale into the
// exponent's multiply-add.
#pragma once
#include "kernels.h"

namespace hydra {

// Positions [lo, hi) of the keys that the query at `pos` sees, or (KEYS) of the queries that see the key at
// `pos`, which lies in one of documents d0 .. d1.  Both ends grow with pos, so a tile's first and last row
// bound what any of its rows sees.
struct Span {
  int lo, hi;
};
template <bool KEYS>
__device__ __forceinline__ Span row_span(const int* __restrict__ cu, const int* __restrict__ pe, int d0, int d1, int pos) {
  int start, end, prefix;
  if (d1 - d0 <= 8) {
    start = ((cint*)cu)[d0];
    end = KEYS ? ((cint*)cu)[d0 + 1] : 0;
    prefix = ((cint*)pe)[d0];
    for (int d = d0 + 1; d <= d1; ++d) {
      const int b = ((cint*)cu)[d], e = KEYS ? ((cint*)cu)[d + 1] : 0, x = ((cint*)pe)[d];
      const bool later = pos >= b;
      start = later ? b : start;
      end = later ? e : end;
      prefix = later ? x : prefix;
    }
  } else {
    int lo = d0, hi = d1 + 1;  // the largest d with cu[d] <= pos
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= pos) lo = mid; else hi = mid;
    }
    start = cu[lo];
    end = cu[lo + 1];
    prefix = pe[lo];
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(start), "+v"(end), "+v"(prefix)::"memory");
  }
  if (KEYS) return {pos < prefix ? start : pos, end};
  return {start, max(pos + 1, prefix)};
}

// What turns raw scores into log2 units, the same for all rows of a head.
struct ScoreConst {
  float sl2;     // softmax scale * log2(e)
  float in;      // softmax scale / cap
  float out;     // cap * log2(e)
  float slope2;  // slope * log2(e)
};
template <int MOD> __device__ __forceinline__ ScoreConst score_const(const Args<MOD>& a, int head) {
  ScoreConst c = {a.scale * LOG2E, 0.f, 0.f, 0.f};
  if constexpr (MOD & kCap) {
    c.in = a.scale / a.cap;
    c.out = a.cap * LOG2E;
  }
  if constexpr (MOD & kBias) c.slope2 = __int_as_float(((cint*)a.slopes)[head]) * LOG2E;
  return c;
}
template <int MOD> constexpr bool in_log2() { return (MOD & (kCap | kBias)) != 0; }

// tanh(x) for |x| <= TANH_NEAR as x P(x^2): the polynomial of least relative error (6e-7) on that range,
// fitted to tanh.  A cap is some ten times the scores it is for, so that blocks of scores beyond it are
// few: the wave takes the exponential form, two quarter-rate instructions an element against none, only
// for those.
constexpr float TANH_NEAR = 0.75f;
__device__ __forceinline__ float tanh_near(float x) {
  const float y = x * x;
  float r = 0.0129296325f;
  r = __builtin_fmaf(r, y, -0.050056303f);
  r = __builtin_fmaf(r, y, 0.132589832f);
  r = __builtin_fmaf(r, y, -0.333282515f);
  r = __builtin_fmaf(r, y, 0.999999435f);
  return x * r;
}
// tanh |x| = 1 - 2 / (e^(2 |x|) + 1), of full relative accuracy beyond TANH_NEAR; infinite x gives 1
__device__ __forceinline__ float tanh_any(float x) {
  const float e = __builtin_amdgcn_exp2f(__builtin_fabsf(x) * (2 * LOG2E));
  const float far = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(e + 1.f), 1.f);
  return __builtin_fabsf(x) > TANH_NEAR ? __builtin_copysignf(far, x) : tanh_near(x);
}

// 16 raw scores -> tanh(s * in)
__device__ __forceinline__ void tanh16(f32x16& s, float in) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 16; e += 2) top = fmax2(fmax2(top, __builtin_fabsf(s[e])), __builtin_fabsf(s[e + 1]));
  if (__builtin_amdgcn_ballot_w64(top * in > TANH_NEAR) != 0) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = tanh_any(s[e] * in);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = tanh_near(s[e] * in);
  }
}

// The bias of an element: its distance is |d0 + DIR * (its offset)|.
template <int DIR> __device__ __forceinline__ float biased(float s, float slope2, float d0, int e) {
  return __builtin_fmaf(-slope2, __builtin_fabsf(d0 + DIR * float(16 * (e >> 3) + (e & 7))), s);
}

// 16 raw scores -> log2 units.
template <int MOD, int DIR> __device__ __forceinline__ void score16(f32x16& s, const ScoreConst& c, float d0) {
  if constexpr (MOD & kCap) {
    tanh16(s, c.in);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] *= c.out;
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] *= c.sl2;
  }
  if constexpr (MOD & kBias) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = biased<DIR>(s[e], c.slope2, d0, e);
  }
}

// The same, and g(e, 1 - tanh^2) for every element of a capped block.
template <int MOD, int DIR, class G>
__device__ __forceinline__ void score16_grad(f32x16& s, const ScoreConst& c, float d0, G&& g) {
  if constexpr (MOD & kCap) {
    tanh16(s, c.in);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      g(e, __builtin_fmaf(-s[e], s[e], 1.f));
      s[e] *= c.out;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] *= c.sl2;
  }
  if constexpr (MOD & kBias) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = biased<DIR>(s[e], c.slope2, d0, e);
  }
}

// f with the variant of a problem's scores as a compile-time number.
template <class F> hipError_t with_mod(const ScoreArgs& a, F&& f) {
  if (a.cap > 0.f) return a.slopes ? f(IntC<kScored | kCap | kBias>{}) : f(IntC<kScored | kCap>{});
  return a.slopes ? f(IntC<kScored | kBias>{}) : f(IntC<kScored>{});
}

}  // namespace hydra
