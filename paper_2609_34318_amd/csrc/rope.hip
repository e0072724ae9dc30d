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

__device__ __forceinline__ u32x4 ld_stream(const char* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
__device__ __forceinline__ void st_stream(char* p, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p)); }

// 8 elements of BYTES bytes each: as they are read, and as 32-bit values.
template <int BYTES> struct Chunk8;
template <> struct Chunk8<2> {
  u32x4 v;
  __device__ __forceinline__ void load(const char* p) { v = ld_stream(p); }
  __device__ __forceinline__ f32x8 wide() const { return widen(v); }
  __device__ __forceinline__ u32x4 bf16() const { return v; }
};
template <> struct Chunk8<4> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const char* p) { a = ld_stream(p), b = ld_stream(p + 16); }
  __device__ __forceinline__ f32x8 wide() const {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
    return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  }
  __device__ __forceinline__ u32x4 bf16() const { return narrow(wide()); }
};

// Element offset of head h of token t: in [G][*] of `width` columns a head, or in token rows.
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

// A lane's chunk of a head, for heads of `chunks` chunks: chunk c of head `sub` of the heads a wave holds.
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

// x rotated: columns [8c, 8c + 8) of a head in this lane, its other chunks in the lanes beside it.
// cs: the token's table; other: LDS column of each column's partner; buf: 64 x 8 floats of this wave.
template <int EX>
__device__ __forceinline__ f32x8 rotate(f32x8 x, const float2* cs, const uint8_t* other, float* buf, int lane,
                                        const LaneMap& m) {
  const int c = m.c;
  const float4* row = reinterpret_cast<const float4*>(cs + 8 * c);
  f32x8 y;
  if constexpr (EX == kInChunk) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
  } else {
    float4* mine = reinterpret_cast<float4*>(buf + 8 * lane);
    wave_lds_order();
    mine[0] = make_float4(x[0], x[1], x[2], x[3]);
    mine[1] = make_float4(x[4], x[5], x[6], x[7]);
    wave_lds_order();
    const float* head = buf + 8 * (m.on ? lane - c : 0);  // the head's first column
    if constexpr (EX == kChunks) {
      const float4* o = reinterpret_cast<const float4*>(head + other[8 * c]);
      const float4 u = o[0], v = o[1];
      y = f32x8{u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = head[other[8 * c + i]];
    }
  }
  f32x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 w = row[i];  // cos, sin of two columns
    r[2 * i] = __builtin_fmaf(x[2 * i], w.x, y[2 * i] * w.y);
    r[2 * i + 1] = __builtin_fmaf(x[2 * i + 1], w.z, y[2 * i + 1] * w.w);
  }
  return r;
}

// LDS of a workgroup: the table, the partners, the waves' exchange buffers.
struct Shared {
  float2* cs;
  uint8_t* other;
  float* buf;
  __device__ __forceinline__ Shared(char* base, const RopeArgs& a, int wave) {
    buf = reinterpret_cast<float*>(base) + wave * 64 * 8;
    other = reinterpret_cast<uint8_t*>(base + kWaves * 64 * 8 * 4);
    cs = reinterpret_cast<float2*>(base + kWaves * 64 * 8 * 4 + kMaxCols);
    for (int j = threadIdx.x; j < a.r.pairs; j += kThreads) {
      other[a.r.first[j]] = a.r.second[j];
      other[a.r.second[j]] = a.r.first[j];
    }
  }
};
size_t shared_bytes(int block_tokens, int cols) {
  return size_t(kWaves) * 64 * 8 * 4 + kMaxCols + size_t(block_tokens) * size_t(cols) * sizeof(float2);
}

// Calls f(t, group of heads) for this wave's share of n tokens x groups.
template <class F> __device__ __forceinline__ void for_items(int wave, int n, int groups, F&& f) {
  int t = wave / groups, hg = wave - t * groups;
  while (t < n) {
    f(t, hg);
    hg += kWaves;
    while (hg >= groups) hg -= groups, ++t;
  }
}

// ------------------------------------------------------------------ queries
// IN_BYTES: of the input's elements.  BWD: [G] -> token rows, else token rows -> [G] (or in place).
template <int EX, int IN_BYTES, bool BWD, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void rope_q_kernel(RopeArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared sh(smem, a, wave);
  const int nope = a.d - a.r.cols;
  for (int64_t t0 = (int64_t)blockIdx.x * a.block_tokens; t0 < a.T; t0 += (int64_t)gridDim.x * a.block_tokens) {
    const int n = (int)min((int64_t)a.block_tokens, a.T - t0);
    __syncthreads();
    fill_table(a, t0, n, sh.cs);
    __syncthreads();
    auto src_at = [&](int64_t t, int h) { return BWD ? at_group(a, t, h, a.d) : t * a.src_stride + (int64_t)h * a.d; };
    auto dst_at = [&](int64_t t, int h) {
      return BWD || IN_PLACE ? t * a.dst_stride + (int64_t)h * a.d : at_group(a, t, h, a.d);
    };
    const LaneMap m(lane, a.r.cols / 8);
    for_items(wave, n, (a.H + m.per_wave - 1) / m.per_wave, [&](int t, int hg) {
      const int h = hg * m.per_wave + m.sub;
      const bool on = m.on && h < a.H;
      Chunk8<IN_BYTES> x{};
      if (on) x.load(a.src + (src_at(t0 + t, h) + nope + 8 * m.c) * IN_BYTES);
      const f32x8 y = rotate<EX>(x.wide(), sh.cs + t * a.r.cols, sh.other, sh.buf, lane, m);
      if (on) st_stream(a.dst + (dst_at(t0 + t, h) + nope + 8 * m.c) * 2, narrow(y));
    });
    if (!IN_PLACE && nope > 0) {
      const LaneMap m2(lane, nope / 8);
      for_items(wave, n, (a.H + m2.per_wave - 1) / m2.per_wave, [&](int t, int hg) {
        const int h = hg * m2.per_wave + m2.sub;
        if (!m2.on || h >= a.H) return;
        Chunk8<IN_BYTES> x;
        x.load(a.src + (src_at(t0 + t, h) + 8 * m2.c) * IN_BYTES);
        st_stream(a.dst + (dst_at(t0 + t, h) + 8 * m2.c) * 2, x.bf16());
      });
    }
  }
}

// ------------------------------------------------------------------ keys and values
template <int EX> __global__ __launch_bounds__(kThreads) void rope_kv_kernel(RopeArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared sh(smem, a, wave);
  const int d_kv = a.d_nope + a.d_v;
  for (int64_t t0 = (int64_t)blockIdx.x * a.block_tokens; t0 < a.T; t0 += (int64_t)gridDim.x * a.block_tokens) {
    const int n = (int)min((int64_t)a.block_tokens, a.T - t0);
    __syncthreads();
    fill_table(a, t0, n, sh.cs);
    __syncthreads();
    // k_pe rotated, to every head
    const LaneMap m(lane, a.r.cols / 8);
    for_items(wave, n, (a.H + m.per_wave - 1) / m.per_wave, [&](int t, int hg) {
      const int h = hg * m.per_wave + m.sub;
      Chunk8<2> x{};
      if (m.on) x.load(a.src2 + ((t0 + t) * a.src2_stride + 8 * m.c) * 2);
      const f32x8 y = rotate<EX>(x.wide(), sh.cs + t * a.r.cols, sh.other, sh.buf, lane, m);
      if (m.on && h < a.H) st_stream(a.dst + (at_group(a, t0 + t, h, a.d) + a.d_nope + 8 * m.c) * 2, narrow(y));
    });
    if (d_kv > 0) {
      const LaneMap m2(lane, d_kv / 8);
      for_items(wave, n, (a.H + m2.per_wave - 1) / m2.per_wave, [&](int t, int hg) {
        const int h = hg * m2.per_wave + m2.sub, col = 8 * m2.c;
        if (!m2.on || h >= a.H) return;
        const u32x4 x = ld_stream(a.src + ((t0 + t) * a.src_stride + (int64_t)h * d_kv + col) * 2);
        if (col < a.d_nope) st_stream(a.dst + (at_group(a, t0 + t, h, a.d) + col) * 2, x);
        else st_stream(a.dst2 + (at_group(a, t0 + t, h, a.d_v) + col - a.d_nope) * 2, x);
      });
    }
  }
}

// The rotation is linear and the same for all heads of a token: their gradients are summed first, then
// rotated back once.  A wave sums a token's heads, its lanes in steps of the heads a wave holds, then over
// those.
template <int EX, int IN_BYTES> __global__ __launch_bounds__(kThreads) void rope_kv_bwd_kernel(RopeArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared sh(smem, a, wave);
  const int d_kv = a.d_nope + a.d_v;
  for (int64_t t0 = (int64_t)blockIdx.x * a.block_tokens; t0 < a.T; t0 += (int64_t)gridDim.x * a.block_tokens) {
    const int n = (int)min((int64_t)a.block_tokens, a.T - t0);
    __syncthreads();
    fill_table(a, t0, n, sh.cs);
    __syncthreads();
    const LaneMap m(lane, a.r.cols / 8);
    for (int t = wave; t < n; t += kWaves) {
      f32x8 sum = {};
      if (m.on)
        for (int h = m.sub; h < a.H; h += m.per_wave) {
          Chunk8<IN_BYTES> x;
          x.load(a.src + (at_group(a, t0 + t, h, a.d) + a.d_nope + 8 * m.c) * IN_BYTES);
          sum += x.wide();
        }
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < 8; ++i) sh.buf[8 * lane + i] = sum[i];
      wave_lds_order();
      if (m.on && m.sub == 0)
        for (int k = 1; k < m.per_wave; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] += sh.buf[8 * (lane + k * (a.r.cols / 8)) + i];
      const f32x8 y = rotate<EX>(sum, sh.cs + t * a.r.cols, sh.other, sh.buf, lane, m);
      if (m.on && m.sub == 0) st_stream(a.dst2 + ((t0 + t) * a.dst2_stride + 8 * m.c) * 2, narrow(y));
    }
    if (d_kv > 0) {
      const LaneMap m2(lane, d_kv / 8);
      for_items(wave, n, (a.H + m2.per_wave - 1) / m2.per_wave, [&](int t, int hg) {
        const int h = hg * m2.per_wave + m2.sub, col = 8 * m2.c;
        if (!m2.on || h >= a.H) return;
        Chunk8<IN_BYTES> x;
        if (col < a.d_nope) x.load(a.src + (at_group(a, t0 + t, h, a.d) + col) * IN_BYTES);
        else x.load(a.src2 + (at_group(a, t0 + t, h, a.d_v) + col - a.d_nope) * IN_BYTES);
        st_stream(a.dst + ((t0 + t) * a.dst_stride + (int64_t)h * d_kv + col) * 2, x.bf16());
      });
    }
  }
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

int check_ptrs(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!p) return HYDRA_ERR_INVALID;
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

// Tokens of a workgroup: as many as give its waves a few wave-sized pieces each, and the table at most
// 16 KB, but 2048 workgroups where there are as many tokens: what one holds in flight does not cover the
// memory's latency.
int block_tokens(int64_t T, int H, int cols) {
  const int groups = (H + 64 / (cols / 8) - 1) / (64 / (cols / 8));
  int n = std::max(1, std::min(32 / groups, 2048 / cols));
  while (n > 1 && T / n < 2048) n /= 2;
  return n;
}

template <class K> int launch(K kernel, const char* name, RopeArgs& a, void* stream) {
  a.block_tokens = block_tokens(a.T, a.H, a.r.cols);
  const int64_t blocks = (a.T + a.block_tokens - 1) / a.block_tokens;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int tok = prof_begin(name, s);
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(kThreads),
                     shared_bytes(a.block_tokens, a.r.cols), s, a);
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
  return ex == kInChunk ? launch(rope_kv_bwd_kernel<kInChunk, IN_BYTES>, "rope_kv_bwd", a, stream)
         : ex == kChunks ? launch(rope_kv_bwd_kernel<kChunks, IN_BYTES>, "rope_kv_bwd", a, stream)
                         : launch(rope_kv_bwd_kernel<kAnywhere, IN_BYTES>, "rope_kv_bwd", a, stream);
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
  if (int rc = check_ptrs({src, positions, dst}); rc != HYDRA_OK) return rc;
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
  if (int rc = check_ptrs({dq, positions, d_src}); rc != HYDRA_OK) return rc;
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
  const void* some = positions;
  if (int rc = check_ptrs({width > 0 ? kv : some, k_pe, positions, k, d_v > 0 ? v : some}); rc != HYDRA_OK) return rc;
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
  const void* some = positions;
  if (int rc = check_ptrs({dk, d_v > 0 ? dv : some, positions, width > 0 ? d_kv : some, d_k_pe}); rc != HYDRA_OK)
    return rc;
  const uint64_t n = uint64_t(n_tokens) * uint64_t(n_heads) * uint64_t(grad_bytes);
  if (any_overlap({{d_kv, width > 0 ? rows_bytes(n_tokens, a.dst_stride, width) : 0},
                   {d_k_pe, rows_bytes(n_tokens, a.dst2_stride, a.r.cols)}},
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
