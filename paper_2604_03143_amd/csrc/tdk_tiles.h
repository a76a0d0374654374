// Building blocks of the attention kernels: tiles of 32 tokens against 32 query rows (v_mfma_f32_32x32x16_bf16), in 64-token steps whose K and V
// rows come from memory straight into LDS, and the step that keeps matrix cores and vector units busy together.
#pragma once

#include "tdk_internal.h"

namespace tdk {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2a __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2a __attribute__((ext_vector_type(2)));

namespace {

constexpr int kTile = 32;            // tokens per MFMA tile
constexpr int kBigTile = 2 * kTile;       // tokens per step of the master pass
constexpr int kVsStride = kHeadDim + 32;  // bf16 elements per staged V row (+64 bytes: four consecutive rows' 64-byte
                                          // pieces then fall into different LDS banks for the transposing reads)

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  f32x2a v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2a));
}

// Running softmax of one query row (the lane pair n, n + 32 shares a row) and its output accumulators:
// oacc[b][i] is element 32 b + 8 (i / 4) + 4 hh + i % 4 of the row's un-normalised output.
struct RowState {
  float m_run, l_run;
  f32x16 oacc[4];
};

// The maximum that goes with a partial sum.  A NaN score keeps a row's reference point at -infinity for as long as no step is
// free of NaN, and the merge takes -infinity for an empty part: such a part says +infinity instead, and the row becomes NaN.
__device__ __forceinline__ float part_max(float m_run, float l_tot) { return m_run == -INFINITY && l_tot != l_tot ? INFINITY : m_run; }

// log-sum-exp of a row: -infinity for an empty one, NaN for a row with a NaN score
__device__ __forceinline__ float row_lse(float m, float l) { return l > 0.f ? m + __logf(l) : l != l ? l : -INFINITY; }

__device__ __forceinline__ void row_state_init(RowState& st) {
  st.m_run = -INFINITY;
  st.l_run = 0.f;
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) st.oacc[b][i] = 0.f;
}

// Orders the LDS traffic of one wavefront (its lanes exchange data through a staging area no other
// wavefront touches): no hardware barrier, only a point the compiler may not move memory accesses across.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The tiles of these kernels: rows of 256 bytes without padding, as the loads that write LDS directly leave them (a wavefront
// instruction fills 1 KB: four rows), with the 16-byte pieces of a row exchanged so that the reads spread over the banks:
// piece c of K row r stands at place c ^ (r % 16) (the score operands of 16 rows fall on all 64 banks), piece c of
// V row r at c ^ 4 (r % 4) (the 64-byte parts of four rows that a transposing read meets do).
constexpr int kStepTile = kBigTile * kHeadDim * 2;        // bytes of one K or V tile of a step
__device__ __forceinline__ int k_place(int r, int c) { return r * (kHeadDim * 2) + 16 * (c ^ (r & 15)); }
__device__ __forceinline__ int v_place(int r, int c) { return r * (kHeadDim * 2) + 16 * (c ^ (4 * (r & 3))); }

// 16 bytes per lane from memory straight into LDS: lane l's piece goes to byte lds + 16 l.  base and lds are the same for
// all lanes.  The instruction writes no register; the compiler does not see that it is in flight: landed() waits for it,
// before the barrier that hands the tile over.  (The builtin makes every later LDS read of the kernel wait for the
// tile, also reads of the other buffer.)  The wait states: M0 before its use, and base, which a vector instruction may
// have written just before.  (M0 has no other use in these kernels, which a test of the assembly pins: the
// compiler reserves M0 and does not take it in the list of registers that a statement overwrites.)
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_byte(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// One thread's share of the loads of a step's tile: thread t brings piece t % 16 of rows t / 16, 16 + t / 16, ...
struct StepLoader {
  uint32_t row_bytes, k_off, v_off;      // distance of two tokens in memory; this thread's places in the first 16 rows
  int st_tok, st_pc;
  uint32_t lds_wave;                     // where this wavefront's four rows of every sixteen go
  __device__ __forceinline__ StepLoader(int heads) {
    st_tok = threadIdx.x >> 4;
    st_pc = threadIdx.x & 15;
    row_bytes = (uint32_t)heads * (kHeadDim * 2);
    k_off = (uint32_t)st_tok * row_bytes + 16u * (st_pc ^ (st_tok & 15));
    v_off = (uint32_t)st_tok * row_bytes + 16u * (st_pc ^ (4 * (st_tok & 3)));
    lds_wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * 1024u;
  }
  // rows 0 .. 63 from `tile` on into the LDS tile at byte `lds`; rows behind `last` repeat that one
  __device__ __forceinline__ void load(const char* tile, int last, uint32_t first, uint32_t lds) const {
    if (last >= kBigTile - 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) load_to_lds(tile + (size_t)(16 * e) * row_bytes, first, lds + 4096u * e + lds_wave);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        load_to_lds(tile, first - (uint32_t)st_tok * row_bytes + (uint32_t)min(16 * e + st_tok, last) * row_bytes, lds + 4096u * e + lds_wave);
    }
  }
};

// maximum of a value over the lane pair (n, n + 32)
__device__ __forceinline__ float pair_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int NT>
__device__ __forceinline__ void rows_max(const f32x16 (&s)[NT], float& mx) {
  mx = s[0][0];
#pragma unroll
  for (int i = 1; i < 16 * NT - 1; i += 2)
    mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(s[i >> 4][i & 15], s[(i + 1) >> 4][(i + 1) & 15]));
  mx = __builtin_elementwise_maximum(mx, s[NT - 1][15]);
}

// mx: each lane's maximum of the masked scores to come (unscaled).  A row's reference point moves when the
// maximum has outgrown it by more than 8.
__device__ __forceinline__ void rows_settle(float mx, float scale, RowState& st) {
  constexpr float kLazy = 8.f;
  const float m = pair_max(mx) * scale;
  if (__any(m > st.m_run + kLazy || (st.m_run == -INFINITY && m != -INFINITY))) {
    const float m_new = m > st.m_run + kLazy || st.m_run == -INFINITY ? fmaxf(st.m_run, m) : st.m_run;
    const float alpha = __expf(st.m_run - (m_new == -INFINITY ? 0.f : m_new));     // 1 for the rows whose reference stays
    st.l_run *= alpha;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.oacc[q][i] *= alpha;
    st.m_run = m_new;
  }
}

// The operands of the two products, from tiles of rows of 256 bytes.  Score product: elements 16 kk + 8 hh .. + 7 of row n
// of the 32 rows from `Ks` on.  Second product: see pv_tr; tokens 16 kk .. + 15, elements 32 q .. + 31.
__device__ __forceinline__ bf16x8 k_operand(const unsigned char* Ks, int kk, int n, int hh) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(Ks + (k_place(n, hh) ^ (32 * kk))));
}
__device__ __forceinline__ bf16x8 v_operand(const unsigned char* Vs, int kk, int q, int lane) {
  const int i16 = lane & 15, blk = lane >> 4;
  const unsigned char* p = Vs + (v_place(4 * (blk >> 1) + (i16 >> 2), 2 * (blk & 1)) ^ (64 * q)) + 8 * (i16 & 3);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (16 * kk) * (kHeadDim * 2)));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (16 * kk + 8) * (kHeadDim * 2)));
  const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
  return __builtin_bit_cast(bf16x8, u32x4{l2.x, l2.y, h2.x, h2.y});
}

__device__ __forceinline__ void rows_scores(const unsigned char* Ks, const bf16x8 (&qf)[8], int n, int hh, f32x16 (&s)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
#pragma unroll
    for (int t = 0; t < 2; ++t)
      s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(Ks + t * (kStepTile / 2), kk, n, hh), qf[kk], s[t], 0, 0, 0);
}

// One pipelined step: the score products of the next step's K tile (16 operands of 32 tokens x 16 elements), the
// weights of this step's scores, and the products of this step's V tile (16 operands of 32 elements x 16 tokens).
// The order is written down slot by slot, because a wavefront only keeps the matrix cores and the vector units
// busy together if their instructions alternate: a slot is the product(s) of one operand, the LDS read of the
// operand four slots ahead, and a few weights (scale and reference point in one fma, exp2, sum, packing), spread so
// that a slot's vector work takes about as long as its products; the maxima of the new scores stand in the last
// slots.  A weight is 2^(scale log2(e) score + reference()).  nx: the raw scores of the next step, mx: their maxima; s is used up.
template <class Reference>
__device__ __forceinline__ void rows_step(const unsigned char* Ks, const unsigned char* Vs, const bf16x8 (&qf)[8], f32x16 (&s)[2],
                                          f32x16 (&nx)[2], float& mx, float scale, int lane, RowState& st, Reference reference) {
  constexpr float kLog2e = 1.4426950408889634f;
  constexpr int kAhead = 4;                                 // (6 and 8 measured the same)
  const int n = lane & 31, hh = lane >> 5;
  const float c2 = scale * kLog2e;
  const float m2 = reference();
  auto k_op = [&](int j) { return k_operand(Ks + (j & 1) * (kStepTile / 2), j >> 1, n, hh); };
  auto v_op = [&](int j) { return v_operand(Vs, j >> 2, j & 3, lane); };
  constexpr int kWeights = 32;
  // weight number w, in the order the second products need them: 16 tokens at a time
  uint32_t pw[4][4];
  // in three stages, each a slot after the one before: a chain of scaling, exponential, sum and packing inside one slot
  // is longer than its product and holds up the next one (12 agents x 2496 tokens x 320 rows 67.6 -> 64.8 us)
  auto tile = [](int w) { return w / 16; };
  auto elem = [](int w) { return 8 * ((w / 8) & 1) + w % 8; };
  auto weight = [&](int w) {
    if (w + 2 < kWeights) s[tile(w + 2)][elem(w + 2)] = __builtin_fmaf(s[tile(w + 2)][elem(w + 2)], c2, m2);
    if (w + 1 < kWeights) s[tile(w + 1)][elem(w + 1)] = __builtin_amdgcn_exp2f(s[tile(w + 1)][elem(w + 1)]);
    st.l_run += s[tile(w)][elem(w)];
    if (w & 1) pw[w / 8][(w % 8) >> 1] = pack2(s[tile(w - 1)][elem(w - 1)], s[tile(w)][elem(w)]);
  };
  // weights before the first product (while its operands arrive), per slot of the first and of the second products;
  // the eight weights of 16 tokens must stand before the four slots that use them
  constexpr int kPre = 4, kFirst = 1, kSecond = 1;
  static_assert(kPre + 16 * kFirst >= 8 && kPre + 16 * kFirst + 4 * kSecond >= 16 && kPre + 16 * kFirst + 8 * kSecond >= 24 &&
                kPre + 16 * kFirst + 12 * kSecond >= 32, "weights stand before their products");
  // The step goes before whatever the unit's other wavefront does between its own steps (tiles, masks, listed pages): with that, and
  // one weight per slot to the end instead of two in the first of the second products, 25 agents x 4992 tokens x 320 rows 196.8
  // -> 191.9 us, x 2496 with a fifth of the pages listed 139.5 -> 131.4.
  __builtin_amdgcn_s_setprio(1);
  bf16x8 ka[kAhead], va[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) ka[j] = k_op(j);
  s[tile(0)][elem(0)] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[tile(0)][elem(0)], c2, m2));
  s[tile(1)][elem(1)] = __builtin_fmaf(s[tile(1)][elem(1)], c2, m2);
#pragma unroll
  for (int w = 0; w < kPre; ++w) weight(w);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    f32x16 c;
    if (j < 2) {
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = 0.f;
    } else {
      c = nx[j & 1];
    }
    nx[j & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[j % kAhead], qf[j >> 1], c, 0, 0, 0);
    if (j + kAhead < 16) ka[j % kAhead] = k_op(j + kAhead);
    else va[j % kAhead] = v_op(j + kAhead - 16);
#pragma unroll
    for (int w = 0; w < kFirst; ++w)
      if (kPre + kFirst * j + w < kWeights) weight(kPre + kFirst * j + w);
    __builtin_amdgcn_sched_barrier(0);
  }
  mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[j >> 2][0], pw[j >> 2][1], pw[j >> 2][2], pw[j >> 2][3]});
    st.oacc[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j % kAhead], pb, st.oacc[j & 3], 0, 0, 0);
    if (j + kAhead < 16) va[j % kAhead] = v_op(j + kAhead);
#pragma unroll
    for (int w = 0; w < kSecond; ++w)
      if (kPre + 16 * kFirst + kSecond * j + w < kWeights) weight(kPre + 16 * kFirst + kSecond * j + w);
    if (j >= 8) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int i = 4 * (j - 8) + 2 * q;
        mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(nx[i >> 4][i & 15], nx[i >> 4][(i & 15) + 1]));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
}
// the same for reference points of scaled scores
__device__ __forceinline__ void rows_step(const unsigned char* Ks, const unsigned char* Vs, const bf16x8 (&qf)[8], f32x16 (&s)[2],
                                          f32x16 (&nx)[2], float& mx, float scale, int lane, RowState& st) {
  rows_step(Ks, Vs, qf, s, nx, mx, scale, lane, st, [&] { return -(st.m_run == -INFINITY ? 0.f : st.m_run) * 1.4426950408889634f; });
}

}  // namespace

}  // namespace tdk
