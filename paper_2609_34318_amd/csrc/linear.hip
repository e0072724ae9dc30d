// Linear attention with a decay for each head (hydra_linear.h).
//
// Every output is one recurrence with the operands changed about.  Over the rows of a sequence, in order or from the
// last to the first,
//   y_i = tx sum over j up to i of L^|i - j| <a_i, b_j> c_j  +  ts (decay since the chunk's edge) a_i S,
// where S collects tu b_j^T c_j, decayed, over the rows before the chunk of i:
//   forward   a, b, c = q, k, v              in order      tx = ts = scale, tu = 1
//   dq        a, b, c = dO, v, k (S^T)       in order      the same
//   dk        a, b, c = v, dO, q (G^T)       from the end  tx = tu = scale, ts = 1
//   dv        a, b, c = k, q, dO (G)         from the end  the same
// A workgroup walks the rows of one item (linear_plan.h) and head in chunks of 32; wave w holds the columns
// 32 w .. 32 w + 31 of S in its accumulators, [d of a] x 32 in 32 bits, through the whole walk.  Per chunk it computes
//   X = b a^T (32 x 32, every wave for itself: sharing it would take an exchange and a barrier), weighted by the decays,
//   y^T = S^T a^T, weighted, + c^T X,
//   S = L^32 S + b^T (weighted c).
// The MFMA result layout is chosen (rows in the order pi, kernels.h) so that X, and S itself, are operands of the next
// products as they lie in the registers; a, b and c come through swizzled LDS tiles, b and c by transpose reads too.
// Later chunks' tiles are copied while one is computed; a wave's rows of y leave through the LDS of its own columns of
// c, so that a chunk has one barrier.
//
// Sequences longer than an item are cut: a first launch (MAIN = false) leaves what each item adds to the state, a scan
// turns that into the states that the items start from, and the main launch walks every item from its own.
//
// Rounding: MFMA operands are bf16.  A weighted c enters the state as a sum of two bf16 values (16 bits), or three (24
// bits) where the walk ends in a state that the caller gets.  X and S enter the products for y as one (each term of y
// then has one rounding of 2^-8 beside the output's own), in the forward as sums of two: what follows o, a norm and
// its gradients, would carry the difference of o from its own rounding further (a layer's gradients off by 3.8e-3 of
// their norm instead of 2.4e-3; forward of 16K rows x 16 heads 74 to 82 us).
//
// 16K rows x 16 heads of 128 x 128 (profiler, 200 passes; rates with the copies of a second read), forward: states 36 us
// (4.6 TB/s; 37 without any computation), scan 15, main 75 (289 MiB, 4.05 TB/s); backward: states 59 (4.8 TB/s), scan 15, main
// 156 (722 MiB, 4.85 TB/s), where a copy of 1 GiB runs at 5.15.  All but one are bound by HBM traffic, some of it beyond the
// algorithm's.  The forward's main launch is not: without computation it takes 39 us (k and v then come from the cache behind
// the L2).  What bounds it is a chunk's chain of dependent work at two waves a SIMD (1.4 on average): the matrix units are
// busy for 32% of the cycles (52 products of 32 cycles a chunk and wave), the vector unit for 49% (some 500 instructions),
// which overlap in part only, and a wave waits for 21% of its time.  (Backward: 35%, 44%, 26%.)  Measured and not kept: three
// waves on a SIMD (registers spill: main 1.4 times slower), priorities around the products and forced orders of products,
// reads and vector work (the same to 2%), deeper copies than the LDS of two workgroups holds at three stages (the same).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <initializer_list>

#include "kernels.h"
#include "linear_plan.h"
#include "plans.h"
#include "prof.h"

namespace hydra {
namespace {

constexpr int LB = 32;  // rows of a chunk

// One walk.  x_g: query heads per head of tensor x; x_s: elements between its token rows.
struct Walk {
  const uint16_t *a, *b, *c;
  int a_s, b_s, c_s, a_g, b_g, c_g;
  const float* in;   // the caller's states that sequences start from, or null
  float* out;        // where their last states go, or null
  float* slots;      // states of cut sequences' items
  int trans;         // the caller's states are [columns of c][columns of a]
  uint16_t* y;       // bf16 [rows][H][columns of c], or
  float* y32;        // fp32; neither: only the last states
  float tx, ts, tu;
};
struct Common {
  const int* items;
  const float* decay;
  int n_items, H;
};

// exp2 arguments are multiples of this: finite, so that no decay times 0 rows is NaN
__device__ __forceinline__ float log2_decay(const float* decay, int head) {
  return fmax2(__int_as_float(((cint*)decay)[head]) * LOG2E, -1.0e30f);
}

// w x, and 0 for x = 0 whatever w: the weights of a short chunk's rows that do not exist (zeros in LDS) may have grown past
// 32 bits where those of its own rows have not.  One instruction, as the product (weights of these rows held at 0 and the
// whole chunks' formed anew behind a short one: up to 37 registers spilled).  The compiler has no builtin for it.
extern "C" __device__ float hydra_fmul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");
__device__ __forceinline__ float weighted(float x, float w) { return hydra_fmul_legacy(x, w); }

// x as bf16, and what that leaves of it (the pairs' bits, so that a value is converted once)
__device__ __forceinline__ bf16x8 split_bf16(float (&x)[8]) {
  const bf16x8 hi = to_bf16x8(x);
  const u32x4 bits = __builtin_bit_cast(u32x4, hi);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] -= __uint_as_float(bits[i] << 16);
    x[2 * i + 1] -= __uint_as_float(bits[i] & 0xffff0000u);
  }
  return hi;
}

template <int DA, int DC, bool MAIN> struct LinGeom {
  static constexpr int WAVES = DC / 32, COPY = WAVES >= 4 ? 4 : 2;  // waves that issue copies
  static constexpr int A = MAIN ? LB * DA * 2 : 0, B = LB * DA * 2, C = LB * DC * 2, STAGE = A + B + C;
  // chunks in LDS, all but one of them on their way: two workgroups run on a CU, with half of its 160 KB each
  static constexpr int STAGES = 4 * STAGE <= 80 << 10 ? 4 : 3 * STAGE <= 80 << 10 ? 3 : 2;
  static constexpr int LDS = STAGES * STAGE;
  static constexpr int COPIES = LB / 8 / COPY * (DA / 64 * (MAIN ? 2 : 1) + DC / 64);  // instructions of a copying wave
};

// Waits for all but the last N vector memory instructions of the wave.
template <int N> __device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// ... of a chunk's copies behind which STAGES - 2 chunks of `copies` are on their way, and the stores of the last T
// chunks' rows (T up to STAGES - 1)
template <int STAGES, int COPIES, int STORES> __device__ __forceinline__ void wait_chunk(int t) {
  constexpr int N = (STAGES - 2) * COPIES;
  if (STORES == 0 || t == 0) wait_vm<N>();
  else if (STAGES == 2 || t == 1) wait_vm<N + STORES>();
  else if (STAGES == 3 || t == 2) wait_vm<N + 2 * STORES>();
  else wait_vm<N + 3 * STORES>();
}

// The lane's part of a 32-column state [DA][32] in the caller's layout.
template <int DA, int DC, class F> __device__ __forceinline__ void each_state(float* p, int trans, int wave, int lane, F&& f) {
  const int m = lane & 31, h = lane >> 5;
#pragma unroll
  for (int b = 0; b < DA / 32; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int da = 32 * b + 16 * (r >> 3) + 8 * h + (r & 7), dc = 32 * wave + m;
      f(b, r, p + (trans ? dc * DA + da : da * DC + dc));
    }
}

// PARTS: bf16 values that a weighted c is cut into.  REST: X and S enter the products for y as two.
template <int DA, int DC, bool REV, bool MAIN, int PARTS, bool REST>
__device__ __forceinline__ void lin_walk(const Walk& w, const Common& cm, int item, int head, lds_char* smem) {
  typedef LinGeom<DA, DC, MAIN> G;
  constexpr int NB = DA / 32;
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (wave >= G::WAVES) return;  // the launch has a wider walk too; ended waves are not waited for at barriers
  const int* it = cm.items + (int64_t)item * LIN_INTS;
  const int row0 = __builtin_amdgcn_readfirstlane(it[LIN_ROW0]), rows = __builtin_amdgcn_readfirstlane(it[LIN_ROWS]);
  const int seq = __builtin_amdgcn_readfirstlane(it[LIN_SEQ]), slot = __builtin_amdgcn_readfirstlane(it[LIN_SLOT]);
  const bool first = __builtin_amdgcn_readfirstlane(it[REV ? LIN_LAST : LIN_FIRST]) != 0;
  const bool last = __builtin_amdgcn_readfirstlane(it[REV ? LIN_FIRST : LIN_LAST]) != 0;
  if (!MAIN && (slot < 0 || last)) return;
  const bool want_y = MAIN && (w.y || w.y32);
  if (MAIN && !want_y && !(last && w.out)) return;

  const float g2 = log2_decay(cm.decay, head);
  auto power = [&](float e) { return __builtin_amdgcn_exp2f(g2 * e); };
  const int n_chunks = (rows + LB - 1) / LB;
  const int a_off = MAIN ? dma_lane_off<DA>(w.a_s, head / w.a_g, wave, lane) : 0;
  const int b_off = dma_lane_off<DA>(w.b_s, head / w.b_g, wave, lane);
  const int c_off = dma_lane_off<DC>(w.c_s, head / w.c_g, wave, lane);
  auto chunk_row = [&](int t) { return LB * (REV ? n_chunks - 1 - t : t); };  // of the item
  auto issue = [&](int t) {
    if (wave >= G::COPY) return;
    const int r = chunk_row(t), n = min(LB, rows - r);
    const int64_t row = row0 + r;
    lds_char* s = smem + (t % G::STAGES) * G::STAGE;
    if constexpr (MAIN) dma_tile<DA, LB, G::COPY>(s, tile_rsrc(w.a, row, n, w.a_s), a_off, w.a_s, wave);
    dma_tile<DA, LB, G::COPY>(s + G::A, tile_rsrc(w.b, row, n, w.b_s), b_off, w.b_s, wave);
    dma_tile<DC, LB, G::COPY>(s + G::A + G::B, tile_rsrc(w.c, row, n, w.c_s), c_off, w.c_s, wave);
  };

  // the state that the item starts from
  auto slot_at = [&](int s) {
    return (char*)(w.slots + ((int64_t)s * cm.H + head) * (DA * DC)) + wave * (DA * 128) + lane * 16;
  };
  const int64_t user = ((int64_t)seq * cm.H + head) * (DA * DC);
  f32x16 S[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) S[b] = f32x16{};
  if (MAIN && slot >= 0) {
    const char* p = slot_at(slot);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(p + (4 * b + rr) * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) S[b][4 * rr + e] = v[e];
      }
  } else if (first && w.in) {
    each_state<DA, DC>(const_cast<float*>(w.in) + user, w.trans, wave, lane, [&](int b, int r, float* p) { S[b][r] = *p; });
  }
  auto store_slot = [&](int s) {
    char* p = slot_at(s);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr)
        *reinterpret_cast<f32x4*>(p + (4 * b + rr) * 1024) =
            f32x4{S[b][4 * rr], S[b][4 * rr + 1], S[b][4 * rr + 2], S[b][4 * rr + 3]};
  };
  // the main launch's first item takes its start from a slot too: the caller's last states may replace the first
  if (!MAIN && first) store_slot(slot);
#pragma unroll
  for (int b = 0; b < NB; ++b) settle(S[b]);

  // weights: of X at this lane's element r, of c at this lane's rows
  float wx[16], wu[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int j = 16 * (r >> 3) + 8 * h + (r & 7), d = REV ? j - m : m - j;
    wx[r] = d < 0 ? 0.f : w.tx * power(float(d));
    wu[r] = w.tu * power(float(REV ? j + 1 : LB - 1 - j));
  }
  const float full_decay = power(float(LB));

  OperandOffsets o = operand_offsets(lane);
  int nat[4];  // as o.b128, of row m
#pragma unroll
  for (int j = 0; j < 4; ++j) nat[j] = m * 128 + (((2 * j + h) ^ swz(m)) << 4);
  int trp[2][2];  // as o.tr, columns in the order pi
  {
    const int g = lane >> 4, gi = lane & 15, x = gi & 3, sw = ((x & 1) << 1) | (x >> 1);
    const int cl = 2 * (g & 1) + (sw >> 1), half = (sw & 1) << 3;
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = 8 * h + (gi >> 2) + 4 * v;
        trp[v][k] = r * 128 + (((4 * k + cl) ^ swz(r)) << 4) + half;
      }
  }
  // transpose reads of the wave's own columns of c
  const int ct0 = (wave >> 1) * block_bytes<LB>() + ((wave & 1) ? o.tr[0][1] : o.tr[0][0]);
  const int ct1 = (wave >> 1) * block_bytes<LB>() + ((wave & 1) ? o.tr[1][1] : o.tr[1][0]);

#pragma unroll
  for (int t = 0; t < G::STAGES - 1; ++t)
    if (t < n_chunks) issue(t);
  float unit = 1.f;
  for (int t = 0; t < n_chunks; ++t) {
    const int r0 = chunk_row(t), n = min(LB, rows - r0);
    lds_char* As = smem + (t % G::STAGES) * G::STAGE;
    lds_char* Bs = As + G::A;
    lds_char* Cs = Bs + G::B;
    // this chunk's copies; later ones' and the stores of earlier rows may be in flight
    if (t + G::STAGES - 2 >= n_chunks) wait_dma();
    else if (!want_y) wait_chunk<G::STAGES, G::COPIES, 0>(t);
    else if (w.y) wait_chunk<G::STAGES, G::COPIES, 2>(t);
    else wait_chunk<G::STAGES, G::COPIES, 4>(t);
    if (n < LB && wave < G::COPY) {
      clear_tail<DA, LB, G::COPY>(Bs, n, wave, lane);
      clear_tail<DC, LB, G::COPY>(Cs, n, wave, lane);
    }
    barrier_lds();
    if (t + G::STAGES - 1 < n_chunks) issue(t + G::STAGES - 1);

    if (!REV && n < LB) {  // an item's last rows
#pragma unroll
      for (int r = 0; r < 16; ++r) wu[r] = w.tu * power(float(max(n - 1 - (16 * (r >> 3) + 8 * h + (r & 7)), 0)));
      asm volatile("" ::: "memory");  // a branch: the compiler would compute both for every chunk
    }
    // S = unit S' of the registers: `unit` alone decays, and S' takes it up only where it leaves 2^-24 .. 2^24
    const float unit0 = unit;
    unit *= n == LB ? full_decay : power(float(n));
    const bool rescale = __builtin_amdgcn_ballot_w64(!(unit > 0x1p-24f && unit < 0x1p24f)) != 0;
    const float new_unit = rescale ? 1.f : unit, per_unit = __builtin_amdgcn_rcpf(new_unit);

    // One block without branches, so that the vector work and the reads lie between the products.
    bf16x8 cf[2];  // c^T: lane = column, rows 16 s + 8 h .. + 7
#pragma unroll
    for (int s = 0; s < 2; ++s) cf[s] = join(lds_tr8(Cs + 2048 * s + ct0), lds_tr8(Cs + 2048 * s + ct1));
    f32x16 x = f32x16{}, y = f32x16{};
    if constexpr (MAIN) {
#pragma unroll
      for (int k = 0; k < DA / 16; ++k) {
        const bf16x8 af = lds_ld16(As, nat[k & 3] + (k >> 2) * block_bytes<LB>());
        x = mfma(op_b128<LB>(Bs, o, 0, k), af, x);
        float s8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s8[e] = S[k >> 1][8 * (k & 1) + e];
        if constexpr (!REST) {
          y = mfma(to_bf16x8(s8), af, y);
        } else {
          y = mfma(split_bf16(s8), af, y);
          y = mfma(to_bf16x8(s8), af, y);
        }
      }
    }
    bf16x8 part[2][PARTS];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float c8[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c8[e] = weighted((float)cf[s][e], wu[8 * s + e] * per_unit);
#pragma unroll
      for (int i = 0; i < PARTS - 1; ++i) part[s][i] = split_bf16(c8);
      part[s][PARTS - 1] = to_bf16x8(c8);
    }
    if (rescale) {
#pragma unroll
      for (int b = 0; b < NB; ++b) S[b] *= unit;
      asm volatile("" ::: "memory");
    }
    unit = new_unit;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const lds_char* q = Bs + (b >> 1) * block_bytes<LB>() + 2048 * s;
        const bf16x8 bf = join(lds_tr8(q + trp[0][b & 1]), lds_tr8(q + trp[1][b & 1]));
#pragma unroll
        for (int i = 0; i < PARTS; ++i) S[b] = mfma(bf, part[s][i], S[b]);
      }

    if (want_y) {
      y *= w.ts * unit0 * power(float(REV ? n - 1 - m : m + 1));
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = weighted(x[8 * s + e], wx[8 * s + e]);
        if constexpr (REST) y = mfma(cf[s], split_bf16(p), y);
        y = mfma(cf[s], to_bf16x8(p), y);
      }
      // rows out through the wave's own columns of c's tile, which no other wave reads: 64 bytes of each row
      const int pitch = cm.H * DC;
      const int64_t at = ((int64_t)(row0 + r0) * cm.H + head) * DC + 32 * wave;
      auto own = [&](int row, int chunk) {
        return Cs + (wave >> 1) * block_bytes<LB>() + row * 128 + (((4 * (wave & 1) + chunk) ^ swz(row)) << 4);
      };
      wave_lds_order();
      if (w.y) {
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
          *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(own(m, rr) + 8 * h) =
              u32x2{pack_bf16x2(y[4 * rr], y[4 * rr + 1]), pack_bf16x2(y[4 * rr + 2], y[4 * rr + 3])};
        wave_lds_order();
        const rows_rsrc ry = rows_buffer(w.y + at, n, pitch * 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = 16 * i + (lane >> 2), ch = lane & 3;
          __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(own(row, ch)), ry,
                                                 row * pitch * 2 + ch * 16, 0, 0);
        }
      } else {  // 32 bits: 16 rows at a time, a row in two rows' places
        const rows_rsrc ry = rows_buffer(w.y32 + at, n, pitch * 4);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if ((m >> 4) == half) {
#pragma unroll
            for (int rr = 0; rr < 4; ++rr)
              *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(own(2 * (m & 15) + (rr >> 1), 2 * (rr & 1) + h)) =
                  f32x4{y[4 * rr], y[4 * rr + 1], y[4 * rr + 2], y[4 * rr + 3]};
          }
          wave_lds_order();
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 8 * i + (lane >> 3), ch = lane & 7;
            __builtin_amdgcn_raw_buffer_store_b128(
                *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(own(2 * row + (ch >> 2), ch & 3)), ry,
                (16 * half + row) * pitch * 4 + ch * 16, 0, 0);
          }
          wave_lds_order();
        }
      }
    }

  }
#pragma unroll
  for (int b = 0; b < NB; ++b) S[b] *= unit;

  if (!MAIN) store_slot(REV ? slot - 1 : slot + 1);
  else if (last && w.out)
    each_state<DA, DC>(w.out + user, w.trans, wave, lane, [&](int b, int r, float* p) { *p = S[b][r]; });
}

template <int DK, int DV, bool MAIN, int PARTS>
__global__ __launch_bounds__(2 * DV) __attribute__((amdgpu_waves_per_eu(2))) void lin_fwd_kernel(Walk w, Common cm) {
  __shared__ __attribute__((aligned(1024))) char smem[LinGeom<DK, DV, MAIN>::LDS];
  lin_walk<DK, DV, false, MAIN, PARTS, true>(w, cm, blockIdx.x / cm.H, blockIdx.x % cm.H, (lds_char*)smem);
}

// The three walks of an item and head run on one XCD (workgroup b runs on XCD b % 8), one after another, and find each
// other's tiles in its L2.  The first launch has two: dk starts from the states of dv, transposed.
template <int DK, int DV, bool MAIN, int PARTS>
__global__ __launch_bounds__(2 * (DK > DV ? DK : DV)) __attribute__((amdgpu_waves_per_eu(2))) void lin_bwd_kernel(Walk dq, Walk dk, Walk dv, Common cm) {
  constexpr int L0 = LinGeom<DV, DK, MAIN>::LDS, L1 = LinGeom<DK, DV, MAIN>::LDS;
  __shared__ __attribute__((aligned(1024))) char smem[L0 > L1 ? L0 : L1];
  constexpr int ROLES = MAIN ? 3 : 2;
  const int j = blockIdx.x / N_XCD, role = j % ROLES, unit = j / ROLES * N_XCD + blockIdx.x % N_XCD;
  const int item = unit / cm.H, head = unit % cm.H;
  if (item >= cm.n_items) return;
  if (role == 0) lin_walk<DV, DK, false, MAIN, 2, false>(dq, cm, item, head, (lds_char*)smem);
  else if (role == 1) lin_walk<DK, DV, true, MAIN, PARTS, false>(dv, cm, item, head, (lds_char*)smem);
  else if constexpr (MAIN) lin_walk<DV, DK, true, MAIN, 2, false>(dk, cm, item, head, (lds_char*)smem);
}

// The states that a cut sequence's items start from, out of what each adds: in order slot s = L^seg slot (s - 1) +
// slot s from the third on (the first holds the start and the second the state behind the first item), from the end
// the same backwards.  One lane walks four elements; eight slots' loads are in flight.  turned: dk walks from the
// transposed states of dv's walk, which are written as it loads them: a block of 32 x 32 is one of 4 KB in both.
struct Scan {
  float *slots, *turned;
  int rev;
};
__global__ __launch_bounds__(256) void lin_scan_kernel(Scan s0, Scan s1, const int* scans, Common cm, int seg, int dk, int dv) {
  const Scan s = blockIdx.z == 0 ? s0 : s1;
  const int scan = blockIdx.y / cm.H, head = blockIdx.y % cm.H, dd = dk * dv;
  const int slot0 = scans[2 * scan], n = scans[2 * scan + 1];
  const int e = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= dd) return;
  const float decay = __builtin_amdgcn_exp2f(log2_decay(cm.decay, head) * float(seg));
  const int64_t step = (int64_t)cm.H * dd * (s.rev ? -1 : 1);
  const int64_t at = ((int64_t)(s.rev ? slot0 + n - 1 : slot0) * cm.H + head) * dd;
  float* p = s.slots + at + e;
  // element (row of dk, column of dv) = (16 (rr / 2) + 8 h + 4 (rr % 2) + 0 .. 3, m) of block (b, w)
  const int w = e / (dk * 32), b = e / 1024 % (dk / 32), rr = e / 256 % 4, lane = e / 4 % 64, m = lane & 31, h = lane >> 5;
  const int row = 16 * (rr >> 1) + 8 * h + 4 * (rr & 1);
  float* q = s.turned ? s.turned + at + b * (dv * 32) + (4 * w + 2 * (m >> 4) + ((m >> 2) & 1)) * 256 +
                            (32 * ((m >> 3) & 1) + row) * 4 + (m & 3)
                      : nullptr;
  auto turn = [&](int i, f32x4 v) {
    if (!q) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) q[i * step + 4 * t] = v[t];
  };
  f32x4 v = *reinterpret_cast<const f32x4*>(p + step);
  turn(0, *reinterpret_cast<const f32x4*>(p));
  turn(1, v);
  constexpr int AHEAD = 8;
  for (int i = 2; i < n; i += AHEAD) {
    f32x4 u[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i + k < n) u[k] = *reinterpret_cast<const f32x4*>(p + (i + k) * step);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i + k < n) {
        v = v * decay + u[k];
        *reinterpret_cast<f32x4*>(p + (i + k) * step) = v;
        turn(i + k, v);
      }
  }
}

// Sums over the query heads of a K/V head: x [rows][Hkv][grp][8 d8] in 32 bits -> y [rows][Hkv][8 d8] bf16, n8 pieces of
// eight; dk, then dv.
struct Group {
  const float* x;
  uint16_t* y;
  int64_t n8;
  int d8;
};
__global__ __launch_bounds__(256) void lin_group_kernel(Group k, Group v, int grp) {
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < k.n8 + v.n8; j += (int64_t)gridDim.x * 256) {
    const bool second = j >= k.n8;
    const int64_t i = second ? j - k.n8 : j;
    const int d8 = second ? v.d8 : k.d8;
    const float* p = (second ? v.x : k.x) + (i / d8 * grp * d8 + i % d8) * 8;
    f32x4 lo = f32x4{}, hi = f32x4{};
    for (int g = 0; g < grp; ++g, p += d8 * 8) {
      lo += *reinterpret_cast<const f32x4*>(p);
      hi += *reinterpret_cast<const f32x4*>(p + 4);
    }
    const float r[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    *reinterpret_cast<bf16x8*>((second ? v.y : k.y) + i * 8) = to_bf16x8(r);
  }
}

// ------------------------------------------------------------------ one token
// A workgroup takes 32 columns of one row's and head's state: lane group r = tid / 8 its rows r, r + 16, ..., lane
// tid % 8 four columns.  Bound by the state's bytes, read and written once in 32 bits (168 rows x 16 heads of 128 x 128:
// 72 us, 5.0 TB/s); columns in four workgroups also spread a single row over 64 CUs.  The first row of a slot takes the
// later ones too, in order, with the state in its registers; a workgroup reads all slots for that, once where no slot is
// there twice: work that grows with the square of the rows (4096 rows x 4 heads of 64 x 64: 115 us, 89 without slots; 1024
// rows: 30 and 29; 64K rows x 1 head: 1.42 ms and 0.44).  A repeated slot's next row is looked for up to the first 1024 rows
// that hold one, so that n rows of one slot are n times the same work (1.2 us each; a search to the last row took 5 of 32K).
constexpr int STEP_THREADS = 128;
template <int DK, int DV>
__global__ __launch_bounds__(STEP_THREADS) void lin_step_kernel(int n_rows, int n_slots, int H, int Hkv, float scale,
                                                                const uint16_t* __restrict__ q, const uint16_t* __restrict__ k,
                                                                const uint16_t* __restrict__ v, const float* __restrict__ decay,
                                                                const float* state, float* state_out,
                                                                const int* __restrict__ slots, uint16_t* __restrict__ o) {
  constexpr int NR = DK / 16;
  __shared__ f32x4 part[2][8];
  __shared__ int next_row[2];
  const int tid = threadIdx.x, r = tid >> 3, c4 = tid & 7;
  const int cb = blockIdx.x % (DV / 32), rest = blockIdx.x / (DV / 32), head = rest % H;
  int row = rest / H;
  const int slot = slots ? slots[row] : row;
  if (slot < 0 || slot >= n_slots) return;
  const int kv = head / (H / Hkv);
  const int64_t at = ((int64_t)slot * H + head) * (DK * DV) + (int64_t)r * DV + 32 * cb + 4 * c4;
  f32x4 S[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) S[i] = *reinterpret_cast<const f32x4*>(state + at + i * 16 * DV);
  constexpr int NO_ROW = 0x7fffffff;
  int next = NO_ROW;  // the slot's next row, of those that this lane looks at
  // f(row) of the rows from `first` on that have the slot, 1024 rows at a time; with `stop` up to the 1024 that have one
  auto each_row = [&](int first, bool stop, auto f) {
    for (int b = first; b < n_rows; b += 8 * STEP_THREADS) {
      int at[8];
      if (b + 8 * STEP_THREADS <= n_rows) {
#pragma unroll
        for (int u = 0; u < 8; ++u) at[u] = slots[b + tid + u * STEP_THREADS];
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) at[u] = b + tid + u * STEP_THREADS < n_rows ? slots[b + tid + u * STEP_THREADS] : -1;
      }
      bool any = false;
#pragma unroll
      for (int u = 0; u < 8; ++u) any |= at[u] == slot;
      if (any) {  // seldom: that row's own and a slot's that is there twice
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (at[u] == slot) f(b + tid + u * STEP_THREADS);
      }
      if (stop && __syncthreads_or(any)) break;
    }
  };
  if (slots) {
    int earlier = 0;
    each_row(0, false, [&](int b) {
      earlier |= b < row;
      if (b > row) next = min(next, b);
    });
    if (__syncthreads_or(earlier)) return;  // not the slot's first row: nothing to do
  }
  const float dec = expf(fmax2(decay[head], -1.0e30f));
  for (;;) {
    const int64_t kq = ((int64_t)row * Hkv + kv) * DK, qq = ((int64_t)row * H + head) * DK;
    const u32x2 vv = *reinterpret_cast<const u32x2*>(v + ((int64_t)row * Hkv + kv) * DV + 32 * cb + 4 * c4);
    const f32x4 v4 = {__uint_as_float(vv[0] << 16), __uint_as_float(vv[0] & 0xffff0000u), __uint_as_float(vv[1] << 16),
                      __uint_as_float(vv[1] & 0xffff0000u)};
    f32x4 sum = f32x4{};
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const float ki = __uint_as_float((uint32_t)k[kq + r + 16 * i] << 16), qi = __uint_as_float((uint32_t)q[qq + r + 16 * i] << 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        S[i][e] = __builtin_fmaf(ki, v4[e], S[i][e] * dec);
        sum[e] = __builtin_fmaf(qi, S[i][e], sum[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum[e] += __shfl_xor(sum[e], 8, 64);
      sum[e] += __shfl_xor(sum[e], 16, 64);
      sum[e] += __shfl_xor(sum[e], 32, 64);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) next = min(next, __shfl_xor(next, d, 64));
    if ((tid & 63) < 8) part[tid >> 6][tid & 7] = sum;
    if ((tid & 63) == 0) next_row[tid >> 6] = next;
    __syncthreads();
    if (tid < 8) {
      const f32x4 t = (part[0][tid] + part[1][tid]) * scale;
      *reinterpret_cast<u32x2*>(o + ((int64_t)row * H + head) * DV + 32 * cb + 4 * tid) =
          u32x2{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
    }
    next = min(next_row[0], next_row[1]);
    if (next == NO_ROW) break;
    row = next;
    next = NO_ROW;
    each_row(row + 1, true, [&](int b) { next = min(next, b); });
    __syncthreads();  // part and next_row are read
  }
#pragma unroll
  for (int i = 0; i < NR; ++i) *reinterpret_cast<f32x4*>(state_out + at + i * 16 * DV) = S[i];
}

// ------------------------------------------------------------------ host side

// f with the head sizes as compile-time numbers.
template <class F> hipError_t with_dims(int dk, int dv, F&& f) {
  if (dv == 64)
    return dk == 64 ? f(IntC<64>{}, IntC<64>{}) : dk == 128 ? f(IntC<128>{}, IntC<64>{}) : f(IntC<192>{}, IntC<64>{});
  return dk == 64 ? f(IntC<64>{}, IntC<128>{}) : dk == 128 ? f(IntC<128>{}, IntC<128>{}) : f(IntC<192>{}, IntC<128>{});
}

struct Timed {
  int tok;
  hipStream_t s;
  Timed(const char* name, hipStream_t st) : tok(prof_begin(name, st)), s(st) {}
  ~Timed() { prof_end(tok, s); }
};

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
bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
uint64_t rows_bytes(int64_t rows, int64_t stride, int64_t width) {
  return rows > 0 ? uint64_t((rows - 1) * stride + width) * 2 : 0;
}

// A checked problem, its plans and its workspace.
struct Plans {
  LinearProblem pr;
  LinearPlan plan[2];  // LinearFor
  LinearLayout w;
  int make(const hydra_linear_t* p) {
    if (int rc = check_linear(p, &pr); rc != HYDRA_OK) return rc;
    linear_plan(pr, LinearFor::kForward, &plan[0]);
    linear_plan(pr, LinearFor::kBackward, &plan[1]);
    w = linear_layout(pr, plan[0], plan[1]);
    return HYDRA_OK;
  }
  int check_workspace(const void* ws, size_t bytes) const {
    if (!ws || bytes < w.total) return HYDRA_ERR_WORKSPACE;
    return misaligned(ws, 16) ? HYDRA_ERR_ALIGN : HYDRA_OK;
  }
  // What a plan depends on; the leading number is no head count of an attention plan's.
  std::vector<int64_t> key() const {
    std::vector<int64_t> k = {-2, pr.H};
    k.insert(k.end(), pr.cu.begin(), pr.cu.end());
    return k;
  }
  int upload(void* ws, hipStream_t s) const {
    hipStreamCaptureStatus recording = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &recording) != hipSuccess) return HYDRA_ERR_HIP;
    if (recording != hipStreamCaptureStatusNone) return HYDRA_ERR_WORKSPACE;  // a replay would copy from a freed image
    std::vector<int32_t> image(w.slots_off / sizeof(int32_t), 0);
    for (int i = 0; i < 2; ++i) {
      std::copy(plan[i].items.begin(), plan[i].items.end(), image.begin() + int64_t(w.items_off[i] / sizeof(int32_t)));
      std::copy(plan[i].scans.begin(), plan[i].scans.end(), image.begin() + int64_t(w.scans_off[i] / sizeof(int32_t)));
    }
    // pageable source: the runtime has consumed the image when the call returns
    if (hipMemcpyAsync(ws, image.data(), image.size() * sizeof(int32_t), hipMemcpyHostToDevice, s) != hipSuccess)
      return HYDRA_ERR_HIP;
    plans_record(ws, key());
    return HYDRA_OK;
  }
  // The workspace holds the plan.
  int ready(bool planned, void* ws, hipStream_t s) const {
    if (!planned) return upload(ws, s);
    return plans_hold(ws, key()) ? HYDRA_OK : HYDRA_ERR_WORKSPACE;
  }
  Common common(LinearFor call, const void* ws, const float* decay) const {
    const int i = int(call);
    return {reinterpret_cast<const int*>(static_cast<const char*>(ws) + w.items_off[i]), decay, plan[i].n_items, pr.H};
  }
  hipError_t scan(LinearFor call, const char* ws, const Common& cm, std::initializer_list<Scan> walks, hipStream_t s) const {
    const Scan* p = walks.begin();
    const int n = int(walks.size()), i = int(call);
    Timed timed("linear_scan", s);
    // a grid's second size ends at 65535
    const int per = std::max(1, 65535 / pr.H);
    for (int at = 0; at < plan[i].n_scans; at += per)
      hipLaunchKernelGGL(lin_scan_kernel, dim3(unsigned(pr.dk * pr.dv / 1024), unsigned(std::min(per, plan[i].n_scans - at) * pr.H), unsigned(n)),
                         dim3(256), 0, s, p[0], p[n > 1 ? 1 : 0], reinterpret_cast<const int*>(ws + w.scans_off[i]) + 2 * at, cm,
                         plan[i].seg, pr.dk, pr.dv);
    return hipGetLastError();
  }
};

int linear_fwd(const hydra_linear_t* p, const void* q, const void* k, const void* v, const float* decay,
               const float* state_in, void* o, float* state_out, void* workspace, size_t bytes, bool planned, void* stream) {
  Plans P;
  if (int rc = P.make(p); rc != HYDRA_OK) return rc;
  const LinearProblem& pr = P.pr;
  const LinearLayout& w = P.w;
  const uint64_t states = uint64_t(pr.cu.size() - 1) * pr.H * pr.dk * pr.dv * 4;
  if (!decay) return HYDRA_ERR_INVALID;
  if (pr.rows > 0 && (!q || !k || !v || (!o && !state_out))) return HYDRA_ERR_INVALID;
  for (const void* x : {q, k, v, static_cast<const void*>(state_in), static_cast<const void*>(o), static_cast<const void*>(state_out)})
    if (misaligned(x, 16)) return HYDRA_ERR_ALIGN;
  if (misaligned(decay, 4)) return HYDRA_ERR_ALIGN;
  if (int rc = P.check_workspace(workspace, bytes); rc != HYDRA_OK) return rc;
  const Span outs[3] = {{o, uint64_t(pr.rows) * pr.H * pr.dv * 2}, {state_out, states}, {workspace, w.total}};
  const Span qs{q, rows_bytes(pr.rows, pr.q_s, pr.H * pr.dk)}, ks{k, rows_bytes(pr.rows, pr.k_s, pr.Hkv * pr.dk)},
      vs{v, rows_bytes(pr.rows, pr.v_s, pr.Hkv * pr.dv)}, ds{decay, uint64_t(pr.H) * 4},
      is{state_in == state_out ? nullptr : state_in, states}, is2{state_in, states};
  if (outputs_overlap({outs[0], outs[1], outs[2]}, {qs, ks, vs, ds, is}) || overlap(outs[0], is2) || overlap(outs[2], is2))
    return HYDRA_ERR_INVALID;
  if (pr.rows == 0 && !state_out) return HYDRA_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (int rc = P.ready(planned, workspace, s); rc != HYDRA_OK) return rc;
  char* ws = static_cast<char*>(workspace);
  const LinearPlan& plan = P.plan[int(LinearFor::kForward)];
  const Common cm = P.common(LinearFor::kForward, ws, decay);
  const int grp = pr.H / pr.Hkv;
  auto u16 = [](const void* x) { return static_cast<const uint16_t*>(x); };
  const Walk walk{u16(q), u16(k), u16(v), pr.q_s, pr.k_s, pr.v_s, 1, grp, grp, state_in, state_out,
                  reinterpret_cast<float*>(ws + w.slots_off), 0, static_cast<uint16_t*>(o), nullptr, pr.scale, pr.scale, 1.f};
  const hipError_t e = with_dims(pr.dk, pr.dv, [&](auto dk_, auto dv_) {
    constexpr int DK = decltype(dk_)::value, DV = decltype(dv_)::value;
    if (plan.n_split > 0) {
      {
        Timed timed("linear_states", s);
        const auto kernel = state_out ? lin_fwd_kernel<DK, DV, false, 3> : lin_fwd_kernel<DK, DV, false, 2>;
        hipLaunchKernelGGL(kernel, dim3(unsigned(plan.n_split) * pr.H), dim3(2 * DV), 0, s, walk, cm);
      }
      if (hipError_t x = P.scan(LinearFor::kForward, ws, cm, {Scan{walk.slots, nullptr, 0}}, s); x != hipSuccess) return x;
    }
    Timed timed("linear_fwd", s);
    const auto kernel = state_out ? lin_fwd_kernel<DK, DV, true, 3> : lin_fwd_kernel<DK, DV, true, 2>;
    hipLaunchKernelGGL(kernel, dim3(unsigned(plan.n_items) * pr.H), dim3(2 * DV), 0, s, walk, cm);
    return hipGetLastError();
  });
  return e == hipSuccess ? HYDRA_OK : HYDRA_ERR_HIP;
}

int linear_bwd(const hydra_linear_t* p, const void* q, const void* k, const void* v, const float* decay,
               const float* state_in, const void* d_o, const float* d_state_out, void* dq, void* dk, void* dv,
               float* d_state_in, void* workspace, size_t bytes, bool planned, void* stream) {
  Plans P;
  if (int rc = P.make(p); rc != HYDRA_OK) return rc;
  const LinearProblem& pr = P.pr;
  const LinearLayout& w = P.w;
  const uint64_t states = uint64_t(pr.cu.size() - 1) * pr.H * pr.dk * pr.dv * 4;
  if (!decay) return HYDRA_ERR_INVALID;
  if (pr.rows > 0 && (!q || !k || !v || !d_o || !dq || !dk || !dv)) return HYDRA_ERR_INVALID;
  for (const void* x : {q, k, v, static_cast<const void*>(state_in), d_o, static_cast<const void*>(d_state_out),
                        static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv),
                        static_cast<const void*>(d_state_in)})
    if (misaligned(x, 16)) return HYDRA_ERR_ALIGN;
  if (misaligned(decay, 4)) return HYDRA_ERR_ALIGN;
  if (int rc = P.check_workspace(workspace, bytes); rc != HYDRA_OK) return rc;
  const uint64_t n = uint64_t(pr.rows);
  if (outputs_overlap({{dq, n * pr.H * pr.dk * 2}, {dk, n * pr.Hkv * pr.dk * 2}, {dv, n * pr.Hkv * pr.dv * 2},
                       {d_state_in, states}, {workspace, w.total}},
                      {{q, rows_bytes(pr.rows, pr.q_s, pr.H * pr.dk)}, {k, rows_bytes(pr.rows, pr.k_s, pr.Hkv * pr.dk)},
                       {v, rows_bytes(pr.rows, pr.v_s, pr.Hkv * pr.dv)}, {decay, uint64_t(pr.H) * 4}, {state_in, states},
                       {d_o, n * pr.H * pr.dv * 2}, {d_state_out, states}}))
    return HYDRA_ERR_INVALID;
  if (pr.rows == 0 && !d_state_in) return HYDRA_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (int rc = P.ready(planned, workspace, s); rc != HYDRA_OK) return rc;
  char* ws = static_cast<char*>(workspace);
  const LinearPlan& plan = P.plan[int(LinearFor::kBackward)];
  const Common cm = P.common(LinearFor::kBackward, ws, decay);
  const int grp = pr.H / pr.Hkv, dos = pr.H * pr.dv;
  const int64_t slots = int64_t(plan.n_split) * pr.H * pr.dk * pr.dv;
  float* at = reinterpret_cast<float*>(ws + w.slots_off);
  auto u16 = [](const void* x) { return static_cast<const uint16_t*>(x); };
  auto out16 = [&](void* x) { return grp > 1 ? nullptr : static_cast<uint16_t*>(x); };
  auto out32 = [&](size_t off) { return grp > 1 ? reinterpret_cast<float*>(ws + off) : nullptr; };
  const Walk wq{u16(d_o), u16(v), u16(k), dos, pr.v_s, pr.k_s, 1, grp, grp, state_in, nullptr, at, 1,
                static_cast<uint16_t*>(dq), nullptr, pr.scale, pr.scale, 1.f};
  const Walk wk{u16(v), u16(d_o), u16(q), pr.v_s, dos, pr.q_s, grp, 1, 1, d_state_out, nullptr, at + slots, 1,
                out16(dk), out32(w.dk_off), pr.scale, 1.f, pr.scale};
  const Walk wv{u16(k), u16(q), u16(d_o), pr.k_s, pr.q_s, dos, grp, 1, 1, d_state_out, d_state_in, at + 2 * slots, 0,
                out16(dv), out32(w.dv_off), pr.scale, 1.f, pr.scale};
  const hipError_t e = with_dims(pr.dk, pr.dv, [&](auto dk_, auto dv_) {
    constexpr int DK = decltype(dk_)::value, DV = decltype(dv_)::value;
    auto grid = [&](int items, int walks) { return dim3(unsigned((int64_t(items) * pr.H + N_XCD - 1) / N_XCD * N_XCD * walks)); };
    const dim3 block(2 * std::max(DK, DV));
    if (plan.n_split > 0) {
      {
        Common first = cm;
        first.n_items = plan.n_split;
        Timed timed("linear_states", s);
        const auto kernel = d_state_in ? lin_bwd_kernel<DK, DV, false, 3> : lin_bwd_kernel<DK, DV, false, 2>;
        hipLaunchKernelGGL(kernel, grid(plan.n_split, 2), block, 0, s, wq, wk, wv, first);
      }
      if (hipError_t x = P.scan(LinearFor::kBackward, ws, cm, {Scan{wq.slots, nullptr, 0}, Scan{wv.slots, wk.slots, 1}}, s); x != hipSuccess)
        return x;
    }
    {
      Timed timed("linear_bwd", s);
      const auto kernel = d_state_in ? lin_bwd_kernel<DK, DV, true, 3> : lin_bwd_kernel<DK, DV, true, 2>;
      hipLaunchKernelGGL(kernel, grid(plan.n_items, 3), block, 0, s, wq, wk, wv, cm);
    }
    if (grp > 1 && pr.rows > 0) {
      Timed timed("linear_groups", s);
      const int64_t nk = pr.rows * pr.Hkv * DK / 8, nv = pr.rows * pr.Hkv * DV / 8;
      hipLaunchKernelGGL(lin_group_kernel, dim3(unsigned(std::min<int64_t>((nk + nv + 255) / 256, 1 << 16))), dim3(256), 0, s,
                         Group{wk.y32, static_cast<uint16_t*>(dk), nk, DK / 8}, Group{wv.y32, static_cast<uint16_t*>(dv), nv, DV / 8}, grp);
    }
    return hipGetLastError();
  });
  return e == hipSuccess ? HYDRA_OK : HYDRA_ERR_HIP;
}

}  // namespace
}  // namespace hydra

using namespace hydra;

extern "C" {

size_t hydra_linear_workspace_size(const hydra_linear_t* p) {
  try {
    Plans P;
    return P.make(p) == HYDRA_OK ? P.w.total : 0;
  } catch (...) {
    return 0;
  }
}

int hydra_linear_plan(const hydra_linear_t* p, void* workspace, size_t workspace_bytes, void* stream) {
  try {
    Plans P;
    if (int rc = P.make(p); rc != HYDRA_OK) return rc;
    if (int rc = P.check_workspace(workspace, workspace_bytes); rc != HYDRA_OK) return rc;
    return P.upload(workspace, static_cast<hipStream_t>(stream));
  } catch (...) {
    return HYDRA_ERR_INVALID;
  }
}

int hydra_linear_fwd(const hydra_linear_t* p, const void* q, const void* k, const void* v, const float* decay,
                     const float* state_in, void* o, float* state_out, void* workspace, size_t workspace_bytes,
                     int32_t planned, void* stream) {
  try {
    return linear_fwd(p, q, k, v, decay, state_in, o, state_out, workspace, workspace_bytes, planned != 0, stream);
  } catch (...) {
    return HYDRA_ERR_INVALID;
  }
}

int hydra_linear_bwd(const hydra_linear_t* p, const void* q, const void* k, const void* v, const float* decay,
                     const float* state_in, const void* d_o, const float* d_state_out, void* dq, void* dk, void* dv,
                     float* d_state_in, void* workspace, size_t workspace_bytes, int32_t planned, void* stream) {
  try {
    return linear_bwd(p, q, k, v, decay, state_in, d_o, d_state_out, dq, dk, dv, d_state_in, workspace, workspace_bytes,
                      planned != 0, stream);
  } catch (...) {
    return HYDRA_ERR_INVALID;
  }
}

int hydra_linear_step(int32_t n_rows, int32_t n_slots, int32_t n_heads, int32_t n_kv_heads, int32_t d_k, int32_t d_v,
                      float scale, const void* q, const void* k, const void* v, const float* decay, const float* state,
                      float* state_out, const int32_t* slots, void* o, void* stream) {
  const int hkv = n_kv_heads == 0 ? n_heads : n_kv_heads;
  if (n_rows < 0 || n_rows > 65536 || n_slots < 0 || n_heads <= 0 || n_heads > 4096) return HYDRA_ERR_INVALID;
  if (hkv < 0 || hkv > n_heads || n_heads % hkv != 0 || d_k <= 0 || d_v <= 0) return HYDRA_ERR_INVALID;
  if ((d_k != 64 && d_k != 128 && d_k != 192) || (d_v != 64 && d_v != 128)) return HYDRA_ERR_UNSUPPORTED;
  if (!(scale - scale == 0.f)) return HYDRA_ERR_INVALID;  // not finite
  if (!slots && n_slots < n_rows) return HYDRA_ERR_INVALID;
  // a dispatch holds fewer than 2^32 lanes
  if (int64_t(n_rows) * n_heads * (d_v / 32) >= (int64_t(1) << 32) / STEP_THREADS) return HYDRA_ERR_INVALID;
  if (n_rows == 0) return HYDRA_OK;
  if (!q || !k || !v || !decay || !state || !state_out || !o) return HYDRA_ERR_INVALID;
  for (const void* x : {q, k, v, static_cast<const void*>(state), static_cast<const void*>(state_out), static_cast<const void*>(o)})
    if (misaligned(x, 16)) return HYDRA_ERR_ALIGN;
  if (misaligned(decay, 4) || misaligned(slots, 4)) return HYDRA_ERR_ALIGN;
  const uint64_t n = uint64_t(n_rows), states = uint64_t(n_slots) * n_heads * d_k * d_v * 4;
  const Span so{state_out, states}, si{state, states}, os{o, n * n_heads * d_v * 2};
  if (outputs_overlap({os, so}, {{q, n * n_heads * d_k * 2}, {k, n * hkv * d_k * 2}, {v, n * hkv * d_v * 2},
                                 {decay, uint64_t(n_heads) * 4}, {slots, n * 4}}) ||
      overlap(os, si) || (state != state_out && overlap(so, si)))
    return HYDRA_ERR_INVALID;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const float sc = scale > 0.f ? scale : 1.0f / sqrtf(float(d_k));
  const hipError_t e = with_dims(d_k, d_v, [&](auto dk_, auto dv_) {
    constexpr int DK = decltype(dk_)::value, DV = decltype(dv_)::value;
    Timed timed("linear_step", s);
    hipLaunchKernelGGL((lin_step_kernel<DK, DV>), dim3(unsigned(n_rows) * unsigned(n_heads) * (DV / 32)), dim3(STEP_THREADS), 0,
                       s, n_rows, n_slots, n_heads, hkv, sc, static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k),
                       static_cast<const uint16_t*>(v), decay, state, state_out, slots, static_cast<uint16_t*>(o));
    return hipGetLastError();
  });
  return e == hipSuccess ? HYDRA_OK : HYDRA_ERR_HIP;
}

}  // extern "C"
