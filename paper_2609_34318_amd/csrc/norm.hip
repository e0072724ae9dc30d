// The norm of every head with an activation or a gate, fused with the exchange's unpack (hydra_norm.h).
//
// Both calls are bound by HBM: forward 6 bytes per element with a gate, backward 10, each read or written once (16K
// tokens x 64 heads of 128, profiler: 155 us, 5.2 TB/s, and 273 us, 5.0 TB/s, sums of weights 5).  A lane
// owns 8 channels (16 bytes) of one head for all of its tokens, so that weight and bias, and in the backward the sums of
// their gradients, stay in its registers; the d / 8 lanes of a head are neighbours in one wave and sum by butterfly.  A
// workgroup has 256 such columns, or where a token has fewer several tokens side by side, and takes every `step`-th
// token, so that workgroups running together read neighbouring rows.  Gradients of weight and bias leave each workgroup
// as one row of partial sums, which a second kernel adds in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "hydra_norm.h"
#include "prof.h"

namespace hydra {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
constexpr int kThreads = 256;
// Tokens of a lane at a time (16K tokens x 64 heads of 128, events around it: backward 274 us, 296 with four, which hold a
// third fewer waves; forward 161 and 166).
constexpr int kUnroll = 2;

__device__ __forceinline__ u32x4 ld_stream(const u32x4* p) { return __builtin_nontemporal_load(p); }
__device__ __forceinline__ void st_stream(u32x4* p, u32x4 v) { __builtin_nontemporal_store(v, p); }

__device__ __forceinline__ f32x8 widen(u32x4 v) {
  f32x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = __uint_as_float(v[i] << 16);
    r[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ u32x4 narrow(f32x8 x) { return __builtin_bit_cast(u32x4, __builtin_convertvector(x, bf16x8v)); }

__device__ __forceinline__ float sum8(f32x8 x) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }

// Sum over a head's lanes, a power of two.
__device__ __forceinline__ float head_sum(float x, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) x += __shfl_xor(x, m, 64);
  return x;
}

// act(t) and its derivative; with e = exp(-|t|) in (0, 1] the sigmoid and one minus it are 1 / (1 + e) and e / (1 + e),
// or the other way round.
template <bool SILU> __device__ __forceinline__ void act(float t, float& a, float& da) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(t) * 1.4426950408889634f);
  const float r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;
  const float s = t >= 0.f ? r : er, om = t >= 0.f ? er : r;
  a = SILU ? t * s : s;
  da = SILU ? s + t * (s * om) : s * om;
}

struct NormArgs {
  const u32x4 *x, *gate, *dy;
  u32x4 *y, *dx, *dgate;
  const float *weight, *bias;
  float* part;        // [steps][2][columns]
  int64_t T;
  int cols8;          // columns of 8 channels: H d / 8
  int side;           // tokens side by side in a workgroup
  int head8;          // d / 8
  int group8;         // columns of a head group
  float inv_d, eps;
};

template <bool BWD, bool GATE, bool CENTER, bool SILU>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  const int sub = a.side > 1 ? threadIdx.x / a.cols8 : 0;
  const int col = a.side > 1 ? threadIdx.x - sub * a.cols8 : blockIdx.y * kThreads + threadIdx.x;
  if (sub >= a.side || col >= a.cols8) return;  // whole heads
  f32x8 w, b, dw = f32x8{}, db = f32x8{};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    w[e] = a.weight ? a.weight[col * 8 + e] : 1.f;
    b[e] = a.bias ? a.bias[col * 8 + e] : 0.f;
  }
  const int group = col / a.group8;
  const u32x4* x = a.x + (int64_t)group * a.T * a.group8 + (col - group * a.group8);
  u32x4* dx = BWD ? a.dx + (x - a.x) : nullptr;
  const int64_t step = (int64_t)gridDim.x * a.side;
  for (int64_t t0 = (int64_t)blockIdx.x * a.side + sub; t0 < a.T; t0 += step * kUnroll) {
    u32x4 vx[kUnroll], vg[kUnroll], vd[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t t = t0 + u * step;
      vx[u] = vg[u] = vd[u] = u32x4{0, 0, 0, 0};
      if (t < a.T) {
        vx[u] = ld_stream(x + t * a.group8);
        if (GATE) vg[u] = ld_stream(a.gate + t * a.cols8 + col);
        if (BWD) vd[u] = ld_stream(a.dy + t * a.cols8 + col);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t t = t0 + u * step;
      f32x8 xc = widen(vx[u]);
      if (CENTER) xc -= head_sum(sum8(xc), a.head8) * a.inv_d;
      const float r = __builtin_amdgcn_rsqf(head_sum(sum8(xc * xc), a.head8) * a.inv_d + a.eps);
      xc *= r;
      const f32x8 z = xc * w + b;
      f32x8 f, df;
      const f32x8 arg = GATE ? widen(vg[u]) : z;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float p, q;
        act<SILU>(arg[e], p, q);
        f[e] = p;
        df[e] = q;
      }
      if (!BWD) {
        if (t < a.T) st_stream(a.y + t * a.cols8 + col, narrow(GATE ? z * f : f));
        continue;
      }
      const f32x8 dy = widen(vd[u]);
      if (GATE && t < a.T) st_stream(a.dgate + t * a.cols8 + col, narrow(dy * z * df));
      const f32x8 dz = dy * (GATE ? f : df);
      dw += dz * xc;  // of a token past the end: dy = 0
      db += dz;
      f32x8 g = dz * w;
      const float along = head_sum(sum8(g * xc), a.head8) * a.inv_d;
      if (CENTER) g -= head_sum(sum8(g), a.head8) * a.inv_d;
      if (t < a.T) st_stream(dx + t * a.group8, narrow((g - xc * along) * r));
    }
  }
  if (!BWD || !a.part) return;
  float* p = a.part + (int64_t)blockIdx.x * 2 * a.cols8 * 8 + col * 8;
  if (a.side > 1) {  // one row of a workgroup: the tokens side by side added in order, lane `sub` the e-th of 16 values
    __shared__ float sums[kThreads * 16];
    const int n = a.cols8, me = sub * n + col;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sums[e * kThreads + me] = dw[e];
      sums[(8 + e) * kThreads + me] = db[e];
    }
    __syncthreads();  // threads without a column have ended
    for (int e = sub; e < 16; e += a.side) {
      float x = 0.f;
      for (int i = 0; i < a.side; ++i) x += sums[e * kThreads + i * n + col];
      p[(e >> 3) * n * 8 + (e & 7)] = x;
    }
    return;
  }
  *reinterpret_cast<f32x8*>(p) = dw;
  *reinterpret_cast<f32x8*>(p + a.cols8 * 8) = db;
}

// d_weight and d_bias: the sums of `rows` partial rows (at most 1024).  A workgroup takes 64 columns, 16 lanes of 4 each
// by 16 rows at a time, and adds the 16 sums in order.
__global__ __launch_bounds__(kThreads) void norm_weights_kernel(const float* __restrict__ part, int rows, int cols,
                                                                float* __restrict__ d_weight, float* __restrict__ d_bias) {
  __shared__ f32x4 sums[16][16];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int per = (cols + 63) / 64, which = blockIdx.x / per;
  const int at = (blockIdx.x % per) * 64 + 4 * c;
  f32x4 s = f32x4{};
  if (at < cols) {
    constexpr int AHEAD = 8;  // loads in flight: one after another 1024 rows take 20 us, so 9
    for (int i0 = r; i0 < rows; i0 += 16 * AHEAD) {
      f32x4 v[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int i = i0 + 16 * k;
        v[k] = i < rows ? *reinterpret_cast<const f32x4*>(part + ((int64_t)i * 2 + which) * cols + at) : f32x4{};
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) s += v[k];
    }
  }
  sums[r][c] = s;
  __syncthreads();
  float* out = which ? d_bias : d_weight;
  if (r > 0 || at >= cols || !out) return;
  for (int i = 1; i < 16; ++i) s += sums[i][c];
  *reinterpret_cast<f32x4*>(out + at) = s;
}

bool sizes_ok(int64_t n_tokens, int32_t n_heads, int32_t d) {
  return n_tokens >= 0 && n_tokens <= (int64_t(1) << 31) && n_heads > 0 && n_heads <= 65536 && d >= 8 && d <= 512 &&
         (d & (d - 1)) == 0;
}

struct Shape {
  int cols8, side, blocks, steps;  // steps: workgroups along the tokens
};
// sums: with partial sums, whose rows a workgroup of few tokens would make many of (2K rows x 8 heads of 256: 30 us with 2
// tokens each).
constexpr int kSumTokens = 8;
Shape shape_of(int64_t T, int32_t H, int32_t d, bool sums) {
  Shape s;
  s.cols8 = H * (d / 8);
  s.side = s.cols8 < kThreads ? kThreads / s.cols8 : 1;
  s.blocks = s.side > 1 ? 1 : (s.cols8 + kThreads - 1) / kThreads;
  const int64_t most = std::max(1, 1024 / s.blocks);
  const int64_t tokens = s.side * (sums ? kSumTokens : 1);
  s.steps = int(std::max<int64_t>(1, std::min<int64_t>(most, (T + tokens - 1) / tokens)));
  return s;
}
size_t part_bytes(const Shape& s) { return size_t(s.steps) * 2 * size_t(s.cols8) * 8 * sizeof(float); }

struct Span {
  const void* p;
  uint64_t n;
};
bool overlap(Span a, Span b) {
  if (!a.p || !b.p || a.n == 0 || b.n == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y + b.n && y < x + a.n;
}
bool outputs_overlap(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (auto o2 = o + 1; o2 != outs.end(); ++o2)
      if (overlap(*o, *o2)) return true;
    for (const Span& i : ins)
      if (overlap(*o, i)) return true;
  }
  return false;
}
bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int check(const hydra_norm_t* p) {
  if (!p || !sizes_ok(p->n_tokens, p->n_heads, p->d) || p->cp_u <= 0 || p->n_heads % p->cp_u != 0) return HYDRA_ERR_INVALID;
  if (p->activation != HYDRA_ACT_SIGMOID && p->activation != HYDRA_ACT_SILU) return HYDRA_ERR_INVALID;
  if (!(p->eps >= 0x1p-126f) || !std::isfinite(p->eps)) return HYDRA_ERR_INVALID;
  return HYDRA_OK;
}

template <bool BWD> void launch(const hydra_norm_t* p, const NormArgs& a, const Shape& sh, hipStream_t s) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(sh.steps), unsigned(sh.blocks)), dim3(kThreads), 0, s, a); };
  const bool silu = p->activation == HYDRA_ACT_SILU;
  if (a.gate && p->center) silu ? go(norm_kernel<BWD, true, true, true>) : go(norm_kernel<BWD, true, true, false>);
  else if (a.gate) silu ? go(norm_kernel<BWD, true, false, true>) : go(norm_kernel<BWD, true, false, false>);
  else if (p->center) silu ? go(norm_kernel<BWD, false, true, true>) : go(norm_kernel<BWD, false, true, false>);
  else silu ? go(norm_kernel<BWD, false, false, true>) : go(norm_kernel<BWD, false, false, false>);
}

NormArgs args_of(const hydra_norm_t* p, const Shape& sh, const void* x, const float* weight, const float* bias, const void* gate) {
  NormArgs a{};
  a.x = static_cast<const u32x4*>(x);
  a.gate = static_cast<const u32x4*>(gate);
  a.weight = weight;
  a.bias = bias;
  a.T = p->n_tokens;
  a.cols8 = sh.cols8;
  a.side = sh.side;
  a.head8 = p->d / 8;
  a.group8 = sh.cols8 / p->cp_u;
  a.inv_d = 1.0f / float(p->d);
  a.eps = p->eps;
  return a;
}

}  // namespace
}  // namespace hydra

using namespace hydra;

extern "C" {

int hydra_unpack_heads_normed(const hydra_norm_t* p, const void* x, const float* weight, const float* bias,
                              const void* gate, void* y, void* stream) {
  if (int rc = check(p); rc != HYDRA_OK) return rc;
  if (p->n_tokens == 0) return HYDRA_OK;
  if (!x || !y) return HYDRA_ERR_INVALID;
  for (const void* q : {x, static_cast<const void*>(weight), static_cast<const void*>(bias), gate, static_cast<const void*>(y)})
    if (misaligned(q)) return HYDRA_ERR_ALIGN;
  const uint64_t cols = uint64_t(p->n_heads) * p->d, n = uint64_t(p->n_tokens) * cols * 2;
  if (outputs_overlap({{y, n}}, {{x, n}, {gate, n}, {weight, cols * 4}, {bias, cols * 4}})) return HYDRA_ERR_INVALID;
  const Shape sh = shape_of(p->n_tokens, p->n_heads, p->d, false);
  NormArgs a = args_of(p, sh, x, weight, bias, gate);
  a.y = static_cast<u32x4*>(y);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int tok = prof_begin("unpack_normed", s);
  launch<false>(p, a, sh, s);
  prof_end(tok, s);
  return hipGetLastError() == hipSuccess ? HYDRA_OK : HYDRA_ERR_HIP;
}

size_t hydra_norm_workspace_size(int64_t n_tokens, int32_t n_heads, int32_t d) {
  return sizes_ok(n_tokens, n_heads, d) ? part_bytes(shape_of(n_tokens, n_heads, d, true)) : 0;
}

int hydra_pack_heads_normed_bwd(const hydra_norm_t* p, const void* x, const float* weight, const float* bias,
                                const void* gate, const void* d_y, void* d_x, void* d_gate, float* d_weight,
                                float* d_bias, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(p); rc != HYDRA_OK) return rc;
  const bool sums = d_weight || d_bias;
  if ((d_weight && !weight) || (d_bias && !bias)) return HYDRA_ERR_INVALID;
  if (p->n_tokens > 0 && (!x || !d_y || !d_x || (gate == nullptr) != (d_gate == nullptr))) return HYDRA_ERR_INVALID;
  for (const void* q : {x, static_cast<const void*>(weight), static_cast<const void*>(bias), gate, d_y,
                        static_cast<const void*>(d_x), static_cast<const void*>(d_gate), static_cast<const void*>(d_weight),
                        static_cast<const void*>(d_bias)})
    if (misaligned(q)) return HYDRA_ERR_ALIGN;
  const Shape sh = shape_of(p->n_tokens, p->n_heads, p->d, sums);
  const size_t need = sums ? part_bytes(sh) : 0;
  if (sums && (!workspace || workspace_bytes < need)) return HYDRA_ERR_WORKSPACE;
  if (sums && misaligned(workspace)) return HYDRA_ERR_ALIGN;
  const uint64_t cols = uint64_t(p->n_heads) * p->d, n = uint64_t(p->n_tokens) * cols * 2;
  if (outputs_overlap({{d_x, n}, {d_gate, n}, {d_weight, cols * 4}, {d_bias, cols * 4}, {sums ? workspace : nullptr, need}},
                      {{x, n}, {gate, n}, {d_y, n}, {weight, cols * 4}, {bias, cols * 4}}))
    return HYDRA_ERR_INVALID;
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormArgs a = args_of(p, sh, x, weight, bias, gate);
  a.dy = static_cast<const u32x4*>(d_y);
  a.dx = static_cast<u32x4*>(d_x);
  a.dgate = static_cast<u32x4*>(d_gate);
  a.part = sums ? static_cast<float*>(workspace) : nullptr;
  if (p->n_tokens > 0) {
    const int tok = prof_begin("pack_normed_bwd", s);
    launch<true>(p, a, sh, s);
    prof_end(tok, s);
    if (hipGetLastError() != hipSuccess) return HYDRA_ERR_HIP;
  }
  if (!sums) return HYDRA_OK;
  const int tok = prof_begin("norm_weights", s);
  const int rows = p->n_tokens > 0 ? sh.steps : 0;
  hipLaunchKernelGGL(norm_weights_kernel, dim3(unsigned((cols + 63) / 64 * 2)), dim3(kThreads), 0, s, a.part, rows, int(cols),
                     d_weight, d_bias);
  prof_end(tok, s);
  return hipGetLastError() == hipSuccess ? HYDRA_OK : HYDRA_ERR_HIP;
}

}  // extern "C"
