// Device-side parts of the modified scores (hydra_scores.h): what a row sees, the cap, the bias.
//
// The kernels hold a 32 x 32 block of raw scores in the MFMA's result registers: element e of a lane is at
// offset 16 (e / 8) + e % 8 from the lane's first key (forward, dQ) or first query (dK/dV).  What is done to
// them is counted in instructions per score: the machine runs these kernels at its power limit (1400 W), where an
// instruction saved is time saved whether or not it was hidden behind the matrix products.
#pragma once
#include "kernels.h"

namespace hydra {

// Positions [lo, hi) of the keys that the query at `pos` sees, or (KEYS) of the queries that see the key at
// `pos`, which lies in one of documents d0 .. d1.  Both ends grow with pos, so a tile's first and last row
// bound what any of its rows sees.  With a window a query also sees the keys before its lo at less than `sinks` from
// its document's start, and of keys hi does not grow: a sink is seen to its document's end (span_min, span_max).
// The window costs what its edges cost: tiles at either end of a row's window evaluate the mask, and a tile of 256 rows
// walks 255 keys more than a row (16K rows x 8 heads, cap 50, window 4096: forward 373 us, 820 TFLOP/s of visible pairs
// against 870 of the whole mask; dK/dV 736, dQ from dS 278).  Below some 500 keys the kernels are bound by their rows:
// accumulators read and written, O in two types (8K rows x 16 heads, window 128: forward 59 us, 45 of it bytes).
struct Span {
  int lo, hi, start;  // start: of the document
};
template <bool KEYS, int MOD>
__device__ __forceinline__ Span row_span(const Args<MOD>& a, int d0, int d1, int pos) {
  const int *__restrict__ cu = a.cu, *__restrict__ pe = a.pe;
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
  if constexpr (MOD & kWindow) {
    if (KEYS) return {pos, pos - start >= a.sinks && end - pos > a.window ? pos + a.window : end, start};
    return {max(start, pos - a.window + 1), pos + 1, start};
  }
  if (KEYS) return {pos < prefix ? start : pos, end, start};
  return {start, max(pos + 1, prefix), start};
}

// The smallest and the largest of a wave's values.
__device__ __forceinline__ int span_min(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = min(x, __shfl_xor(x, d, 64));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int span_max(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = max(x, __shfl_xor(x, d, 64));
  return __builtin_amdgcn_readfirstlane(x);
}

// The sinks of a wave's rows, whose documents start at `first` to `last` (n = 0: none, or no rows).
struct Sinks {
  int n, first, last;
  __device__ __forceinline__ bool touch(int kpos, int kn) const { return n > 0 && kpos - last < n && kpos + kn > first; }
};
template <int MOD> __device__ __forceinline__ Sinks wave_sinks(const Args<MOD>& a, int start, bool rows) {
  if constexpr (MOD & kWindow)
    return {rows ? a.sinks : 0, __builtin_amdgcn_readfirstlane(start), __builtin_amdgcn_readlane(start, 31)};
  return {0, 0, 0};
}

// The slope of a head in log2 units, finite: an infinite one times the distance 0 of a row's own key is NaN.
template <int MOD> __device__ __forceinline__ float slope_log2(const Args<MOD>& a, int head) {
  if constexpr (MOD & kBias)
    return __builtin_amdgcn_fmed3f(__int_as_float(((cint*)a.slopes)[head]) * LOG2E, -0x1.fffffep127f, 0x1.fffffep127f);
  return 0.f;
}
template <int MOD> constexpr bool in_log2() { return (MOD & (kCap | kBias)) != 0; }  // the forward's scores

// The factor from what the backward has of a score (raw, or with a cap its tanh) to log2 units.
template <int MOD> __device__ __forceinline__ float log2_unit(const Args<MOD>& a) {
  if constexpr (MOD & kCap) return a.cap_log2;
  else return a.scale * LOG2E;
}

// out * tanh(s * scale / cap) of raw scores s: out is cap * log2(e) in the forward, whose scores are then in log2
// units, and 1 in the backward, which needs 1 - tanh^2 and has a multiply-add for the exponent (16K rows x 8 heads,
// recompute backward: in log2 units there too 1.3% slower).  tanh(x) / x is a polynomial in x^2 of least
// relative error, with the caps and the scale in its coefficients: of three (4e-7) up to |s| = small (TANH_SMALL
// caps), of five (6e-7) up to |s| = near (TANH_NEAR caps).  A cap is some ten times the scores it is for, so most
// blocks of 32 x 32 take the first (forward 840 us with the second alone, 773 with both; dK/dV 1623 and 1533), and
// few the exponential form beyond near, two quarter-rate instructions an element: tanh |x| =
// 1 - 2 / (e^(2 |x|) + 1), of full relative accuracy there; infinite scores give the cap.  Four elements at a time,
// whose chains of dependent instructions fill each other's latency.
// (The functions take any kernel's arguments, so that a plain kernel's discarded branches compile.)
struct CapConst {
  float c4, c3, c2, c1, c0, out;
  // opaque: an instruction reads one scalar register, and the compiler keeps a copy of every second constant
  // in a vector register through the tile loop
  __device__ __forceinline__ explicit CapConst(const ScoreArgs& a)
      : c4(a.poly[4]), c3(a.poly[3]), c2(a.poly[2]), c1(a.poly[1]), c0(a.poly[0]), out(a.out) {
    asm volatile("" : "+s"(c3), "+s"(out));
  }
};
// The polynomials of s[e0 .. e0 + 3].
template <class A> __device__ __forceinline__ void cap_small4(const f32x16& s, int e0, const A& a, float (&r)[4]) {
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = s[e0 + i] * s[e0 + i];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(a.low[2], w[i], a.low[1]);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(r[i], w[i], a.low[0]);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] *= s[e0 + i];
}
__device__ __forceinline__ void cap_near4(const f32x16& s, int e0, const CapConst& c, float (&r)[4]) {
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = s[e0 + i] * s[e0 + i];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(c.c4, w[i], c.c3);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(r[i], w[i], c.c2);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(r[i], w[i], c.c1);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_fmaf(r[i], w[i], c.c0);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] *= s[e0 + i];
}
// The exponential form where |x| is beyond near, else r.
template <class A> __device__ __forceinline__ float cap_far(float x, float r, const A& a, const CapConst& c) {
  const float y = __builtin_amdgcn_exp2f(__builtin_fabsf(x) * a.two_in);
  float z = __builtin_fmaf(-2.f * c.out, __builtin_amdgcn_rcpf(y + 1.f), c.out);
  settle(z);  // computed for every lane: a branch around it would be taken element by element
  return __builtin_fabsf(x) > a.near ? __builtin_copysignf(z, x) : r;
}
// A wave's blocks of 16 scores a lane, in place, masked ones among them.  A lane that holds a NaN (a masked pair whose
// products overflow to infinities of both signs) takes the general form, for it may hold any score besides.
// TIGHT: element groups one after another, for a kernel that has no registers for more.
template <bool TIGHT, int N, class A> __device__ __forceinline__ void cap_blocks(f32x16* s, const A& a) {
  float top[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    top[n] = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e += 2)
      top[n] = fmax2(fmax2(top[n], __builtin_fabsf(s[n][e])), __builtin_fabsf(s[n][e + 1]));
  }
  float t = top[0];
#pragma unroll
  for (int n = 1; n < N; ++n) t = fmax2(t, top[n]);
  if (__builtin_amdgcn_ballot_w64(!(t <= a.small)) == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e0 = 0; e0 < 16; e0 += 4) {
        float r[4];
        cap_small4(s[n], e0, a, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][e0 + i] = r[i];
      }
    return;
  }
  const CapConst c(a);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const bool far = __builtin_amdgcn_ballot_w64(!(top[n] <= a.near)) != 0;
#pragma unroll
    for (int e0 = 0; e0 < 16; e0 += 4) {
      float r[4];
      cap_near4(s[n], e0, c, r);
      if (far) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = cap_far(s[n][e0 + i], r[i], a, c);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][e0 + i] = r[i];
      if constexpr (TIGHT) sched_fence();
    }
  }
}

// weight * x, and 0 where the weight is 0 whatever x is: a masked pair's weight is 0, and its tanh, and so the
// factor 1 - tanh^2 in x, may be NaN.  One instruction like a product (16K rows x 8 heads, dK/dV: 1544 us; 1592 with the
// factor selected by the mask, 1542 without either).  The compiler has no builtin for it.
extern "C" __device__ float hydra_fmul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float mul_zero(float weight, float x) { return hydra_fmul_legacy(weight, x); }

// s with the bias of an element, whose distance is |d0 + DIR * (its offset)|.
template <int DIR> __device__ __forceinline__ float biased(float s, float slope, float d0, int e) {
  return __builtin_fmaf(-slope, __builtin_fabsf(d0 + DIR * float(16 * (e >> 3) + (e & 7))), s);
}

// 16 raw scores -> log2 units with the bias, in groups one after another.
template <int DIR> __device__ __forceinline__ void biased16(f32x16& s, float unit, float slope, float d0) {
#pragma unroll
  for (int e0 = 0; e0 < 16; e0 += 4) {
#pragma unroll
    for (int e = e0; e < e0 + 4; ++e) s[e] = biased<DIR>(s[e] * unit, slope, d0, e);
    sched_fence();
  }
}

// The last factor of a gradient, whose P and dS are 2^P_LOG2 times their values (exact).
template <int MOD> __host__ __device__ constexpr float unscaled(float scale) {
  return MOD == kPlain ? scale : scale * 0x1p-15f;
}
static_assert(P_LOG2 == 15.f, "unscaled");

// Eight 32-bit values -> fp16, round to nearest even, in the registers of an operand fragment.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bf16x8 to_f16x8(const float* v) {
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  const f32x8 x = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  return __builtin_bit_cast(bf16x8, __builtin_convertvector(x, f16x8));
}

// f with the variant of a problem's scores as a compile-time number.
template <int MASK, class F> hipError_t with_mask(const ScoreArgs& a, F&& f) {
  if (a.out > 0.f) return a.slopes ? f(IntC<MASK | kCap | kBias>{}) : f(IntC<MASK | kCap>{});
  return a.slopes ? f(IntC<MASK | kBias>{}) : f(IntC<MASK>{});
}
template <class F> hipError_t with_mod(const ScoreArgs& a, F&& f) {
  return a.window > 0 ? with_mask<kScored | kWindow>(a, f) : with_mask<kScored>(a, f);
}

}  // namespace hydra
