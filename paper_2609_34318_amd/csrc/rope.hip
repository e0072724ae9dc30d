// Rotary positions with several axes, fused with the split and concatenation of an MLA head and with the
// layout of the exchange (hydra_rope.h).
//
// All four calls are bound by HBM bandwidth: every element is read once and written once (2 bytes each
// way forward; backward 4 or 2 read, 2 written).  A workgroup takes a block of tokens.  It forms the
// block's cos and sin once, into LDS, for all heads: the angle in turns, p f / 2 pi, is a product of 64-bit
// fixed point whose integer turns fall off the top, so that far positions lose nothing, and what is
// left is a 32-bit fraction of a turn.  Then its waves move 16-byte chunks (8 columns): a lane keeps one
// chunk of a head throughout, and a wave holds as many whole heads as fit its 64 lanes, so that no lane
// divides an index and a pair's two columns lie in one wave.  Where they lie in one lane (interleaved
// pairs) nothing is exchanged; else the lanes of a wave exchange through LDS of their own.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "hydra_rope.h"
#include "kernels.h"
#include "prof.h"

namespace hydra {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxCols = 2 * HYDRA_ROPE_MAX_PAIRS;

// The rotation as a kernel argument, by column of the r.
struct RopeTable {
  uint64_t freq[HYDRA_ROPE_MAX_PAIRS];  // f / 2 pi, modulo 1, times 2^64
  uint8_t axis[HYDRA_ROPE_MAX_PAIRS];
  uint8_t first[HYDRA_ROPE_MAX_PAIRS], second[HYDRA_ROPE_MAX_PAIRS];  // columns of the pair
  int32_t pairs, cols;
};

// Where a pair's other column lies: in the same chunk, in another chunk at the same place, or anywhere.
enum Exchange { kInChunk, kChunks, kAnywhere };

struct RopeArgs {
  RopeTable r;
  const int* pos;           // [n_axes][T]
  const char *src, *src2;   // q | kv, k_pe | dq | dk, dv
  char *dst, *dst2;
  int64_t T, src_stride, src2_stride, dst_stride, dst2_stride;  // token rows, elements (0: [G])
  int H, g, d, d_nope, d_v; // g: heads of a send buffer
  int block_tokens;
  float sign;               // 1, or -1 for the inverse rotation
};

typedef float f32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x8 widen(u32x4 v) {
  f32x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = __uint_as_float(v[i] << 16);
    r[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ u32x4 narrow(f32x8 x) { return __builtin_bit_cast(u32x4, __builtin_convertvector(x, bf16x8)); }

// Loads leave their lines in the caches, where the kernel before often left them (1021 tokens x 64 heads 12 to 17 us
// a call, 15 to 21 with the non-temporal hint; the same for tensors beyond the caches).
__device__ __forceinline__ u32x4 ld_chunk(const char* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ void st_stream(char* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}

// One lane's chunk: 16 bytes of input, so that a wave's loads are contiguous, 8 columns of bf16 or 4 of fp32.
// As it is read, as 32-bit values, and as the bf16 that is stored.
template <int BYTES> struct Chunk;
template <> struct Chunk<2> {
  static constexpr int N = 8;
  typedef f32x8 Wide;
  u32x4 v;
  __device__ __forceinline__ void load(const char* p) { v = ld_chunk(p); }
  __device__ __forceinline__ Wide wide() const { return widen(v); }
  __device__ __forceinline__ void store(char* p) const { st_stream(p, v); }
  static __device__ __forceinline__ void store(char* p, Wide x) { st_stream(p, narrow(x)); }
};
template <> struct Chunk<4> {
  static constexpr int N = 4;
  typedef f32x4 Wide;
  u32x4 v;
  __device__ __forceinline__ void load(const char* p) { v = ld_chunk(p); }
  __device__ __forceinline__ Wide wide() const { return __builtin_bit_cast(f32x4, v); }
  __device__ __forceinline__ void store(char* p) const { store(p, wide()); }
  static __device__ __forceinline__ void store(char* p, Wide x) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4)),
                                reinterpret_cast<u32x2*>(p));
  }
};

// Element offset of head h of token t in [G][*] of `width` columns a head.
__device__ __forceinline__ int64_t at_group(const RopeArgs& a, int64_t t, int h, int width) {
  const int j = (unsigned)h / (unsigned)a.g;
  return ((j * a.T + t) * a.g + (h - j * a.g)) * width;
}

// cos and signed sin of every column, for tokens [t0, t0 + n): out = x cos + x_other sin.
__device__ __forceinline__ void fill_table(const RopeArgs& a, int64_t t0, int n, float2* cs) {
  for (int i = threadIdx.x; i < n * a.r.pairs; i += kThreads) {
    const int t = i / a.r.pairs, j = i - t * a.r.pairs;
    const int p = a.pos[a.r.axis[j] * a.T + t0 + t];
    const uint64_t f = a.r.freq[j];
    const uint32_t u = p < 0 ? 0u - (uint32_t)p : (uint32_t)p;
    const uint32_t frac = __umulhi((uint32_t)f, u) + (uint32_t)(f >> 32) * u;  // of |p| f / 2 pi, times 2^32
    float s, c;
    sincospif((float)(int32_t)frac * 0x1p-31f, &s, &c);
    s = p < 0 ? -a.sign * s : a.sign * s;
    cs[t * a.r.cols + a.r.first[j]] = make_float2(c, -s);
    cs[t * a.r.cols + a.r.second[j]] = make_float2(c, s);
  }
}

// A lane's chunk of a head, for heads of `chunks` chunks (at most 64): chunk c of head `sub` of the heads a
// wave holds.
struct LaneMap {
  int per_wave, sub, c;
  bool on;
  __device__ __forceinline__ LaneMap(int lane, int chunks) {
    per_wave = 64 / chunks;
    on = lane < per_wave * chunks;
    sub = on ? lane / chunks : 0;
    c = on ? lane - sub * chunks : 0;
  }
};

// x rotated: columns [N c, N c + N) of a head in this lane, its other chunks in the lanes beside it.
// cs: the token's table; other: each column's partner; buf: 64 x N floats of this wave.
template <int EX, int N, class V>
__device__ __forceinline__ V rotate(V x, const float2* cs, const uint8_t* other, float* buf, int lane, const LaneMap& m) {
  const float4* row = reinterpret_cast<const float4*>(cs + N * m.c);
  V y;
  if constexpr (EX == kInChunk) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = x[i ^ 1];
  } else {
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<float4*>(buf + N * lane + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    wave_lds_order();
    const float* head = buf + N * (m.on ? lane - m.c : 0);  // the head's first column
    const int col = N * m.c;
    if constexpr (EX == kChunks) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const float4 u = *reinterpret_cast<const float4*>(head + other[col] + i);
        y[i] = u.x;
        y[i + 1] = u.y;
        y[i + 2] = u.z;
        y[i + 3] = u.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = head[other[col + i]];
    }
  }
  V r;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float4 w = row[i];  // cos, sin of two columns
    r[2 * i] = __builtin_fmaf(x[2 * i], w.x, y[2 * i] * w.y);
    r[2 * i + 1] = __builtin_fmaf(x[2 * i + 1], w.z, y[2 * i + 1] * w.w);
  }
  return r;
}

// LDS of a workgroup: the waves' exchange buffers, the partners, the table, and for sums over heads
// `sums` times cols floats a token.
struct Shared {
  float* buf;
  uint8_t* other;
  float2* cs;
  float* part;
  __device__ __forceinline__ Shared(char* base, const RopeArgs& a, int wave) {
    buf = reinterpret_cast<float*>(base) + wave * 64 * 8;
    other = reinterpret_cast<uint8_t*>(base + kWaves * 64 * 8 * 4);
    cs = reinterpret_cast<float2*>(base + kWaves * 64 * 8 * 4 + kMaxCols);
    part = reinterpret_cast<float*>(cs + a.block_tokens * a.r.cols);
    for (int j = threadIdx.x; j < a.r.pairs; j += kThreads) {
      other[a.r.first[j]] = a.r.second[j];
      other[a.r.second[j]] = a.r.first[j];
    }
  }
};
size_t shared_bytes(int block_tokens, int cols, int sums) {
  return size_t(kWaves) * 64 * 8 * 4 + kMaxCols + size_t(block_tokens) * size_t(cols) * sizeof(float2) +
         size_t(block_tokens) * size_t(sums) * size_t(cols) * sizeof(float);
}

// Calls f(t, group of heads, whether it is one) for this wave's share of n tokens x groups, two at a time (f is
// called by every lane, for loads of both before a use).
template <class F> __device__ __forceinline__ void for_items(int wave, int n, int groups, F&& f) {
  int t = wave / groups, hg = wave - t * groups;
  auto next = [&]() {
    hg += kWaves;
    while (hg >= groups) hg -= groups, ++t;
  };
  while (t < n) {
    const int t0 = t, hg0 = hg;
    next();
    f(t0, hg0, t, hg, t < n);
    next();
  }
}

// Moves chunks of `cols` columns a head, IN_BYTES an element, for n tokens from t0 on: at(t, j, k, col) gives the
// element offsets {source, destination} and the two bases of head k of send buffer j.  A thread's
// chunks are kThreads apart in the order [token][buffer][head][chunk], found by carrying, not by dividing.
template <int IN_BYTES, class F>
__device__ __forceinline__ void move_chunks(const RopeArgs& a, int n, int cols, F&& at) {
  typedef Chunk<IN_BYTES> C;
  constexpr int U = 4;
  const int chunks = cols / C::N, cp_u = a.H / a.g;
  auto split = [&](int i, int& t, int& j, int& k, int& c) {
    int q = i / chunks;
    c = i - q * chunks;
    int r = q / a.g;
    k = q - r * a.g;
    t = r / cp_u;
    j = r - t * cp_u;
  };
  int t, j, k, c, dt, dj, dk, dc;
  split(threadIdx.x, t, j, k, c);
  split(kThreads, dt, dj, dk, dc);
  while (t < n) {
    C x[U];
    char* to[U];
    bool on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      on[u] = t < n;
      if (on[u]) {
        const char* from;
        at(t, j, k, c * C::N, from, to[u]);
        x[u].load(from);
      }
      c += dc;
      k += dk;
      if (c >= chunks) c -= chunks, ++k;
      j += dj;
      if (k >= a.g) k -= a.g, ++j;
      t += dt;
      if (j >= cp_u) j -= cp_u, ++t;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (on[u]) x[u].store(to[u]);
  }
}

// The blocks of tokens of a workgroup: f(first token, tokens), with the table of cos and sin filled.
template <class F> __device__ __forceinline__ void for_blocks(const RopeArgs& a, const Shared& sh, F&& f) {
  for (int64_t t0 = (int64_t)blockIdx.x * a.block_tokens; t0 < a.T; t0 += (int64_t)gridDim.x * a.block_tokens) {
    const int n = (int)min((int64_t)a.block_tokens, a.T - t0);
    __syncthreads();
    fill_table(a, t0, n, sh.cs);
    __syncthreads();
    f(t0, n);
  }
}

// ------------------------------------------------------------------ queries
// IN_BYTES: of the input's elements.  BWD: [G] -> token rows, else token rows -> [G] (or in place).
template <int EX, int IN_BYTES, bool BWD, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void rope_q_kernel(RopeArgs a) {
  typedef Chunk<IN_BYTES> C;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared sh(smem, a, wave);
  const int nope = a.d - a.r.cols;
  for_blocks(a, sh, [&](int64_t t0, int n) {
    auto src_at = [&](int64_t t, int h) { return BWD ? at_group(a, t, h, a.d) : t * a.src_stride + (int64_t)h * a.d; };
    auto dst_at = [&](int64_t t, int h) {
      return BWD || IN_PLACE ? t * a.dst_stride + (int64_t)h * a.d : at_group(a, t, h, a.d);
    };
    const LaneMap m(lane, a.r.cols / C::N);
    const int col = nope + C::N * m.c;
    for_items(wave, n, (a.H + m.per_wave - 1) / m.per_wave, [&](int ta, int ga, int tb, int gb, bool b_on) {
      const int ha = ga * m.per_wave + m.sub, hb = gb * m.per_wave + m.sub;
      const bool on_a = m.on && ha < a.H, on_b = b_on && m.on && hb < a.H;
      C x{}, z{};
      if (on_a) x.load(a.src + (src_at(t0 + ta, ha) + col) * IN_BYTES);
      if (on_b) z.load(a.src + (src_at(t0 + tb, hb) + col) * IN_BYTES);
      const auto y = rotate<EX, C::N>(x.wide(), sh.cs + ta * a.r.cols, sh.other, sh.buf, lane, m);
      if (on_a) C::store(a.dst + (dst_at(t0 + ta, ha) + col) * 2, y);
      if (!b_on) return;  // uniform over the wave
      const auto w = rotate<EX, C::N>(z.wide(), sh.cs + tb * a.r.cols, sh.other, sh.buf, lane, m);
      if (on_b) C::store(a.dst + (dst_at(t0 + tb, hb) + col) * 2, w);
    });
    if (!IN_PLACE && nope > 0)
      move_chunks<IN_BYTES>(a, n, nope, [&](int t, int j, int k, int c, const char*& from, char*& to) {
        const int64_t row = (int64_t)(j * a.g + k) * a.d + c, packed = ((j * a.T + t0 + t) * a.g + k) * a.d + c;
        from = a.src + (BWD ? packed : (t0 + t) * a.src_stride + row) * IN_BYTES;
        to = a.dst + (BWD ? (t0 + t) * a.dst_stride + row : packed) * 2;
      });
  });
}

// ------------------------------------------------------------------ keys and values
template <int EX> __global__ __launch_bounds__(kThreads) void rope_kv_kernel(RopeArgs a) {
  typedef Chunk<2> C;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared sh(smem, a, wave);
  const int d_kv = a.d_nope + a.d_v;
  for_blocks(a, sh, [&](int64_t t0, int n) {
    // k_pe rotated, to every head
    const LaneMap m(lane, a.r.cols / C::N);
    for_items(wave, n, (a.H + m.per_wave - 1) / m.per_wave, [&](int ta, int ga, int tb, int gb, bool b_on) {
      const int ha = ga * m.per_wave + m.sub, hb = gb * m.per_wave + m.sub;
      C x{}, z{};
      if (m.on) x.load(a.src2 + ((t0 + ta) * a.src2_stride + 8 * m.c) * 2);
      if (m.on && b_on) z.load(a.src2 + ((t0 + tb) * a.src2_stride + 8 * m.c) * 2);
      const auto y = rotate<EX, 8>(x.wide(), sh.cs + ta * a.r.cols, sh.other, sh.buf, lane, m);
      if (m.on && ha < a.H) C::store(a.dst + (at_group(a, t0 + ta, ha, a.d) + a.d_nope + 8 * m.c) * 2, y);
      if (!b_on) return;  // uniform over the wave
      const auto w = rotate<EX, 8>(z.wide(), sh.cs + tb * a.r.cols, sh.other, sh.buf, lane, m);
      if (m.on && hb < a.H) C::store(a.dst + (at_group(a, t0 + tb, hb, a.d) + a.d_nope + 8 * m.c) * 2, w);
    });
    if (d_kv > 0)
      move_chunks<2>(a, n, d_kv, [&](int t, int j, int k, int c, const char*& from, char*& to) {
        from = a.src + ((t0 + t) * a.src_stride + (int64_t)(j * a.g + k) * d_kv + c) * 2;
        const int64_t head = (j * a.T + t0 + t) * a.g + k;
        to = c < a.d_nope ? a.dst + (head * a.d + c) * 2 : a.dst2 + (head * a.d_v + c - a.d_nope) * 2;
      });
  });
}

// The rotation is linear and the same for all heads of a token: their gradients are summed first, then
// rotated back once.  One walk over dk does both: a thread keeps one chunk of a head's d columns and takes the
// heads in steps of those that the workgroup holds at once (with few heads several tokens); it stores the chunk
// or, of the rotated columns, adds it up.  Read in a walk of their own, those columns came at 2.8 TB/s
// where the others came at 4.9 (16K tokens x 128 heads, fp32: 716 and 859 us).  The threads' sums are added in LDS; which
// thread adds which heads goes by the sizes of a head and their number alone, not by the launch.
struct SumMap {
  int per_block, heads, tokens;  // heads that a workgroup holds at once: of one token, tokens
  __host__ __device__ SumMap(int chunks, int H) {
    per_block = kThreads / chunks;
    heads = per_block < H ? per_block : H;
    tokens = per_block / heads;
  }
};
template <int EX, int IN_BYTES> __global__ __launch_bounds__(kThreads) void rope_kv_bwd_kernel(RopeArgs a) {
  typedef Chunk<IN_BYTES> C;
  typedef typename C::Wide Wide;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared sh(smem, a, wave);
  const int d_kv = a.d_nope + a.d_v, chunks = a.d / C::N;
  const SumMap m(chunks, a.H);
  const int sub = threadIdx.x / chunks, c = threadIdx.x - sub * chunks, tok = sub / m.heads, first = sub - tok * m.heads;
  const bool sums = c * C::N >= a.d_nope;
  const int step_k = m.heads % a.g;
  const int64_t wrap = (a.T - 1) * a.g * (int64_t)a.d * IN_BYTES;  // from one buffer's end to the next's start
  const int64_t step = (int64_t)m.heads * a.d * IN_BYTES + (m.heads / a.g) * wrap;
  for_blocks(a, sh, [&](int64_t t0, int n) {
    for (int t = tok; t < n; t += m.tokens) {
      if (tok >= m.tokens) break;
      Wide sum = {};
      int k = first % a.g;
      const char* from = a.src + (at_group(a, t0 + t, first, a.d) + c * C::N) * IN_BYTES;
      char* to = a.dst + ((t0 + t) * a.dst_stride + (int64_t)first * d_kv + c * C::N) * 2;
      for (int h = first; h < a.H;) {
        constexpr int U = 2;
        C x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (h + u * m.heads < a.H) x[u].load(from);
          from += step;
          k += step_k;
          if (k >= a.g) k -= a.g, from += wrap;
        }
        if (sums) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (h + u * m.heads < a.H) sum += x[u].wide();
        } else {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (h + u * m.heads < a.H) x[u].store(to + (int64_t)u * m.heads * d_kv * 2);
        }
        to += (int64_t)U * m.heads * d_kv * 2;
        h += U * m.heads;
      }
      if (sums) {
#pragma unroll
        for (int e = 0; e < C::N; ++e) sh.part[(t * m.heads + first) * a.r.cols + c * C::N - a.d_nope + e] = sum[e];
      }
    }
    if (a.d_v > 0)
      move_chunks<IN_BYTES>(a, n, a.d_v, [&](int t, int j, int k, int col, const char*& from, char*& to) {
        from = a.src2 + (((j * a.T + t0 + t) * a.g + k) * a.d_v + col) * IN_BYTES;
        to = a.dst + ((t0 + t) * a.dst_stride + (int64_t)(j * a.g + k) * d_kv + a.d_nope + col) * 2;
      });
    __syncthreads();
    // a wave's lanes take the rotated columns of as many tokens as fit
    const LaneMap l(lane, a.r.cols / C::N);
    for (int i = wave * l.per_wave; i < n; i += kWaves * l.per_wave) {
      const int t = i + l.sub;
      const bool on = l.on && t < n;
      Wide sum = {};
      for (int w = 0; w < (on ? m.heads : 0); ++w)
#pragma unroll
        for (int e = 0; e < C::N; ++e) sum[e] += sh.part[(t * m.heads + w) * a.r.cols + C::N * l.c + e];
      const Wide y = rotate<EX, C::N>(sum, sh.cs + min(t, n - 1) * a.r.cols, sh.other, sh.buf, lane, l);
      if (on) C::store(a.dst2 + ((t0 + t) * a.dst2_stride + C::N * l.c) * 2, y);
    }
  });
}

// ------------------------------------------------------------------ host side
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

struct Span {
  const void* p;
  uint64_t n;
};
bool overlap(Span a, Span b) {
  if (!a.p || !b.p || a.n == 0 || b.n == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y + b.n && y < x + a.n;
}

// f / 2 pi modulo 1, times 2^64 (modulo 2^64).  1 / 2 pi in two doubles, the product's rounding error from a
// fused multiply-add; the error's part may be negative, and wraps like all else.
uint64_t turns64(double f) {
  if (f < 0) return 0 - turns64(-f);  // 1 - a small part would round
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
  const double t = f * hi, e = std::fma(f, hi, -t) + f * lo;
  return uint64_t((t - std::floor(t)) * 0x1p64) + uint64_t(int64_t(e * 0x1p64));
}

// Token rows (bytes): two views of one buffer, of the same stride, overlap only where their columns do.
struct Rows {
  const void* p;
  uint64_t rows, stride, width;
  Span span() const { return {p, rows > 0 && width > 0 ? (rows - 1) * stride + width : 0}; }
};
bool overlap(const Rows& a, const Rows& b) {
  if (!overlap(a.span(), b.span())) return false;
  if (a.stride != b.stride) return true;
  const uint64_t ab = reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p);
  const uint64_t d = ab >> 63 ? (a.stride - (0 - ab) % a.stride) % a.stride : ab % a.stride;  // b's column in a's rows
  return !(a.width <= d && d + b.width <= a.stride);
}

// Checks and fills the table; *ex: how its pairs are exchanged.
int make_table(const hydra_rope_t* r, RopeTable* t, Exchange* ex) {
  if (!r || r->n_axes < 1 || r->n_axes > HYDRA_ROPE_MAX_AXES) return HYDRA_ERR_INVALID;
  if (r->pairing < HYDRA_ROPE_INTERLEAVED || r->pairing > HYDRA_ROPE_AXIS_HALVES) return HYDRA_ERR_INVALID;
  if (r->per_axis != 0 && r->per_axis != 1) return HYDRA_ERR_INVALID;
  if (!r->inv_freq && !(std::isfinite(r->base) && r->base >= 1.0)) return HYDRA_ERR_INVALID;
  int n = 0;
  for (int a = 0; a < r->n_axes; ++a) {
    if (r->pairs[a] < 1 || r->pairs[a] > HYDRA_ROPE_MAX_PAIRS) return HYDRA_ERR_INVALID;
    n += r->pairs[a];
  }
  if (n > HYDRA_ROPE_MAX_PAIRS || n % 4 != 0) return HYDRA_ERR_INVALID;
  *t = RopeTable{};
  t->pairs = n;
  t->cols = 2 * n;
  bool chunks = true;  // both columns of every pair at the same place of a chunk
  int j0 = 0;
  for (int a = 0; a < r->n_axes; ++a) {
    for (int j = j0; j < j0 + r->pairs[a]; ++j) {
      const double f = r->inv_freq   ? r->inv_freq[j]
                       : r->per_axis ? std::pow(r->base, -double(j - j0) / r->pairs[a])
                                     : std::pow(r->base, -double(j) / n);
      if (!(std::fabs(f) <= 0x1p20)) return HYDRA_ERR_INVALID;
      t->freq[j] = turns64(f);
      t->axis[j] = uint8_t(a);
      const int c0 = r->pairing == HYDRA_ROPE_INTERLEAVED ? 2 * j : r->pairing == HYDRA_ROPE_HALVES ? j : j0 + j;
      const int c1 = r->pairing == HYDRA_ROPE_INTERLEAVED ? c0 + 1 : c0 + (r->pairing == HYDRA_ROPE_HALVES ? n : r->pairs[a]);
      t->first[j] = uint8_t(c0);
      t->second[j] = uint8_t(c1);
    }
    if (r->pairing == HYDRA_ROPE_AXIS_HALVES && r->pairs[a] % 8 != 0) chunks = false;
    j0 += r->pairs[a];
  }
  if (r->pairing == HYDRA_ROPE_HALVES && n % 8 != 0) chunks = false;
  *ex = r->pairing == HYDRA_ROPE_INTERLEAVED ? kInChunk : chunks ? kChunks : kAnywhere;
  return HYDRA_OK;
}

// Token rows of `width` elements: their stride (0: dense).
bool row_stride(int64_t s, int64_t width, int64_t* out) {
  if (s == 0) s = width;
  *out = s;
  return s >= width && s % 8 == 0 && s < (int64_t(1) << 30);
}
uint64_t rows_bytes(int64_t rows, int64_t stride, int64_t width) { return uint64_t((rows - 1) * stride + width) * 2; }

int check_sizes(int64_t T, int H, int cp_u) {
  if (T < 0 || T > (int64_t(1) << 30) || H <= 0 || H > 4096 || cp_u <= 0 || H % cp_u != 0) return HYDRA_ERR_INVALID;
  return HYDRA_OK;
}

int check_ptrs(const int32_t* positions, std::initializer_list<const void*> ps) {
  if (!positions) return HYDRA_ERR_INVALID;
  for (const void* p : ps)
    if (!p) return HYDRA_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(positions) % sizeof(int32_t) != 0) return HYDRA_ERR_ALIGN;
  for (const void* p : ps)
    if (!aligned16(p)) return HYDRA_ERR_ALIGN;
  return HYDRA_OK;
}

bool any_overlap(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (auto p = o + 1; p != outs.end(); ++p)
      if (overlap(*o, *p)) return true;
    for (const Span& i : ins)
      if (overlap(*o, i)) return true;
  }
  return false;
}

// Tokens of a workgroup: as few as give its waves two wave-sized pieces of rotated columns each (the fewer, the
// more workgroups of a CU are in different phases: 16K tokens x 128 heads in one token a workgroup against
// two: rope_kv 446 and 486 us, rope_kv_bwd 654 and 719; 32K x 16 heads in four against eight 115 and 127, 184 and
// 187) and a thread an angle to form (64K x 2 heads in eight against four 45 and 59, 65 and 80); but 2048 workgroups
// where there are as many tokens.
int block_tokens(int64_t T, int H, int cols) {
  const int groups = (H + 64 / (cols / 8) - 1) / (64 / (cols / 8));
  int n = std::max(1, std::min(8 / groups, 512 / cols));
  while (n > 1 && T / n < 2048) n /= 2;
  return n;
}

template <class K> int launch(K kernel, const char* name, RopeArgs& a, void* stream, int sums = 0) {
  a.block_tokens = block_tokens(a.T, a.H, a.r.cols);
  const int64_t blocks = (a.T + a.block_tokens - 1) / a.block_tokens;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int tok = prof_begin(name, s);
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(kThreads),
                     shared_bytes(a.block_tokens, a.r.cols, sums), s, a);
  prof_end(tok, s);
  return hipGetLastError() == hipSuccess ? HYDRA_OK : HYDRA_ERR_HIP;
}

template <int IN_BYTES, bool BWD, bool IN_PLACE> int launch_q(Exchange ex, const char* name, RopeArgs& a, void* stream) {
  return ex == kInChunk ? launch(rope_q_kernel<kInChunk, IN_BYTES, BWD, IN_PLACE>, name, a, stream)
         : ex == kChunks ? launch(rope_q_kernel<kChunks, IN_BYTES, BWD, IN_PLACE>, name, a, stream)
                         : launch(rope_q_kernel<kAnywhere, IN_BYTES, BWD, IN_PLACE>, name, a, stream);
}
int launch_kv(Exchange ex, RopeArgs& a, void* stream) {
  return ex == kInChunk ? launch(rope_kv_kernel<kInChunk>, "rope_kv", a, stream)
         : ex == kChunks ? launch(rope_kv_kernel<kChunks>, "rope_kv", a, stream)
                         : launch(rope_kv_kernel<kAnywhere>, "rope_kv", a, stream);
}
template <int IN_BYTES> int launch_kv_bwd(Exchange ex, RopeArgs& a, void* stream) {
  const int sums = SumMap(a.d / Chunk<IN_BYTES>::N, a.H).heads;
  return ex == kInChunk ? launch(rope_kv_bwd_kernel<kInChunk, IN_BYTES>, "rope_kv_bwd", a, stream, sums)
         : ex == kChunks ? launch(rope_kv_bwd_kernel<kChunks, IN_BYTES>, "rope_kv_bwd", a, stream, sums)
                         : launch(rope_kv_bwd_kernel<kAnywhere, IN_BYTES>, "rope_kv_bwd", a, stream, sums);
}

}  // namespace
}  // namespace hydra

using namespace hydra;

extern "C" {

int hydra_rope_q(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_head, int32_t cp_u,
                 const void* src, int64_t src_tok_stride, const int32_t* positions, void* dst, void* stream) {
  RopeArgs a{};
  Exchange ex;
  if (int rc = make_table(r, &a.r, &ex); rc != HYDRA_OK) return rc;
  if (int rc = check_sizes(n_tokens, n_heads, cp_u); rc != HYDRA_OK) return rc;
  if (d_head < a.r.cols || d_head > 512 || d_head % 8 != 0) return HYDRA_ERR_INVALID;
  const int64_t width = int64_t(n_heads) * d_head;
  if (!row_stride(src_tok_stride, width, &a.src_stride)) return HYDRA_ERR_INVALID;
  if (n_tokens == 0) return HYDRA_OK;
  if (int rc = check_ptrs(positions, {src, dst}); rc != HYDRA_OK) return rc;
  const bool in_place = src == dst;
  if (in_place && cp_u != 1) return HYDRA_ERR_INVALID;
  const Span s = {src, rows_bytes(n_tokens, a.src_stride, width)};
  const Span p = {positions, uint64_t(n_tokens) * uint64_t(r->n_axes) * 4};
  const Span d = {dst, in_place ? s.n : uint64_t(n_tokens) * uint64_t(width) * 2};
  if (overlap(d, p) || (!in_place && overlap(d, s))) return HYDRA_ERR_INVALID;
  a.pos = positions;
  a.src = static_cast<const char*>(src);
  a.dst = static_cast<char*>(dst);
  a.T = n_tokens;
  a.dst_stride = a.src_stride;
  a.H = n_heads;
  a.g = n_heads / cp_u;
  a.d = d_head;
  a.sign = 1.f;
  return in_place ? launch_q<2, false, true>(ex, "rope_q", a, stream) : launch_q<2, false, false>(ex, "rope_q", a, stream);
}

int hydra_rope_q_bwd(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_head, int32_t cp_u,
                     int32_t grad_bytes, const void* dq, const int32_t* positions, void* d_src, int64_t src_tok_stride,
                     void* stream) {
  RopeArgs a{};
  Exchange ex;
  if (int rc = make_table(r, &a.r, &ex); rc != HYDRA_OK) return rc;
  if (int rc = check_sizes(n_tokens, n_heads, cp_u); rc != HYDRA_OK) return rc;
  if (d_head < a.r.cols || d_head > 512 || d_head % 8 != 0) return HYDRA_ERR_INVALID;
  if (grad_bytes != 2 && grad_bytes != 4) return HYDRA_ERR_INVALID;
  const int64_t width = int64_t(n_heads) * d_head;
  if (!row_stride(src_tok_stride, width, &a.dst_stride)) return HYDRA_ERR_INVALID;
  if (n_tokens == 0) return HYDRA_OK;
  if (int rc = check_ptrs(positions, {dq, d_src}); rc != HYDRA_OK) return rc;
  if (any_overlap({{d_src, rows_bytes(n_tokens, a.dst_stride, width)}},
                  {{dq, uint64_t(n_tokens) * uint64_t(width) * uint64_t(grad_bytes)},
                   {positions, uint64_t(n_tokens) * uint64_t(r->n_axes) * 4}}))
    return HYDRA_ERR_INVALID;
  a.pos = positions;
  a.src = static_cast<const char*>(dq);
  a.dst = static_cast<char*>(d_src);
  a.T = n_tokens;
  a.H = n_heads;
  a.g = n_heads / cp_u;
  a.d = d_head;
  a.sign = -1.f;
  return grad_bytes == 4 ? launch_q<4, true, false>(ex, "rope_q_bwd", a, stream)
                         : launch_q<2, true, false>(ex, "rope_q_bwd", a, stream);
}

int hydra_rope_kv(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_nope, int32_t d_v, int32_t cp_u,
                  const void* kv, int64_t kv_tok_stride, const void* k_pe, int64_t pe_tok_stride,
                  const int32_t* positions, void* k, void* v, void* stream) {
  RopeArgs a{};
  Exchange ex;
  if (int rc = make_table(r, &a.r, &ex); rc != HYDRA_OK) return rc;
  if (int rc = check_sizes(n_tokens, n_heads, cp_u); rc != HYDRA_OK) return rc;
  if (d_nope < 0 || d_v < 0 || d_nope % 8 != 0 || d_v % 8 != 0 || d_nope > 512 || d_v > 512 || d_nope + d_v > 512 ||
      d_nope + a.r.cols > 512)
    return HYDRA_ERR_INVALID;
  const int64_t width = int64_t(n_heads) * (d_nope + d_v);
  if (!row_stride(kv_tok_stride, width, &a.src_stride) || !row_stride(pe_tok_stride, a.r.cols, &a.src2_stride))
    return HYDRA_ERR_INVALID;
  if (n_tokens == 0) return HYDRA_OK;
  // what is empty needs no address
  if (int rc = check_ptrs(positions, {width > 0 ? kv : k_pe, k_pe, k, d_v > 0 ? v : k_pe}); rc != HYDRA_OK) return rc;
  const uint64_t n = uint64_t(n_tokens) * uint64_t(n_heads) * 2;
  if (any_overlap({{k, n * uint64_t(d_nope + a.r.cols)}, {d_v > 0 ? v : nullptr, n * uint64_t(d_v)}},
                  {{kv, width > 0 ? rows_bytes(n_tokens, a.src_stride, width) : 0},
                   {k_pe, rows_bytes(n_tokens, a.src2_stride, a.r.cols)},
                   {positions, uint64_t(n_tokens) * uint64_t(r->n_axes) * 4}}))
    return HYDRA_ERR_INVALID;
  a.pos = positions;
  a.src = static_cast<const char*>(kv);
  a.src2 = static_cast<const char*>(k_pe);
  a.dst = static_cast<char*>(k);
  a.dst2 = static_cast<char*>(v);
  a.T = n_tokens;
  a.H = n_heads;
  a.g = n_heads / cp_u;
  a.d = d_nope + a.r.cols;
  a.d_nope = d_nope;
  a.d_v = d_v;
  a.sign = 1.f;
  return launch_kv(ex, a, stream);
}

int hydra_rope_kv_bwd(const hydra_rope_t* r, int64_t n_tokens, int32_t n_heads, int32_t d_nope, int32_t d_v,
                      int32_t cp_u, int32_t grad_bytes, const void* dk, const void* dv, const int32_t* positions,
                      void* d_kv, int64_t kv_tok_stride, void* d_k_pe, int64_t pe_tok_stride, void* stream) {
  RopeArgs a{};
  Exchange ex;
  if (int rc = make_table(r, &a.r, &ex); rc != HYDRA_OK) return rc;
  if (int rc = check_sizes(n_tokens, n_heads, cp_u); rc != HYDRA_OK) return rc;
  if (d_nope < 0 || d_v < 0 || d_nope % 8 != 0 || d_v % 8 != 0 || d_nope > 512 || d_v > 512 || d_nope + d_v > 512 ||
      d_nope + a.r.cols > 512)
    return HYDRA_ERR_INVALID;
  if (grad_bytes != 2 && grad_bytes != 4) return HYDRA_ERR_INVALID;
  const int64_t width = int64_t(n_heads) * (d_nope + d_v);
  if (!row_stride(kv_tok_stride, width, &a.dst_stride) || !row_stride(pe_tok_stride, a.r.cols, &a.dst2_stride))
    return HYDRA_ERR_INVALID;
  if (n_tokens == 0) return HYDRA_OK;
  if (int rc = check_ptrs(positions, {dk, d_v > 0 ? dv : dk, width > 0 ? d_kv : dk, d_k_pe}); rc != HYDRA_OK) return rc;
  const uint64_t n = uint64_t(n_tokens) * uint64_t(n_heads) * uint64_t(grad_bytes);
  const Rows kv_rows = {d_kv, uint64_t(n_tokens), uint64_t(a.dst_stride) * 2, uint64_t(width) * 2};
  const Rows pe_rows = {d_k_pe, uint64_t(n_tokens), uint64_t(a.dst2_stride) * 2, uint64_t(a.r.cols) * 2};
  if (overlap(kv_rows, pe_rows)) return HYDRA_ERR_INVALID;
  for (const Span& out : {kv_rows.span(), pe_rows.span()})
    if (any_overlap({out},
                  {{dk, n * uint64_t(d_nope + a.r.cols)},
                   {d_v > 0 ? dv : nullptr, n * uint64_t(d_v)},
                   {positions, uint64_t(n_tokens) * uint64_t(r->n_axes) * 4}}))
    return HYDRA_ERR_INVALID;
  a.pos = positions;
  a.src = static_cast<const char*>(dk);
  a.src2 = static_cast<const char*>(dv);
  a.dst = static_cast<char*>(d_kv);
  a.dst2 = static_cast<char*>(d_k_pe);
  a.T = n_tokens;
  a.H = n_heads;
  a.g = n_heads / cp_u;
  a.d = d_nope + a.r.cols;
  a.d_nope = d_nope;
  a.d_v = d_v;
  a.sign = -1.f;
  return grad_bytes == 4 ? launch_kv_bwd<4>(ex, a, stream) : launch_kv_bwd<2>(ex, a, stream);
}

}  // extern "C"
