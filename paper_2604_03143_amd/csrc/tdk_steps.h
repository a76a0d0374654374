// Attention of many query rows to tokens that come in steps of 64: four wavefronts of 32 rows share tiles of K and V in LDS, one barrier a step; the scores of
// the next step stand beside the weights and second products of this one, and what is behind them travels meanwhile.  A Source brings the
// tiles: rows as they are (tdk_prompt_attend.hip), or pages in 8 bits (tdk_kv8.hip).
#pragma once

#include "tdk_kv_pages.h"

namespace tdk {

namespace {

constexpr int kStep = kBigTile;              // tokens of a step
constexpr int kRows = 4 * 32;                // query rows of a workgroup, 32 per wavefront

struct StepTiles {
  unsigned char k[2][kStepTile];
  unsigned char v[2][kStepTile];
  int odd[2][4];                             // per V tile and wavefront: it holds infinity or NaN that only some rows may meet
  uint8_t marks[kRows][kHeadDim / 2];        // of that, what each row has met, by element (four bits each): bit 0 +infinity, 1 -infinity, 2 NaN
};

// bits of two bf16 values, four each
__device__ __forceinline__ uint32_t odd_kinds(uint32_t w) {
  const auto kind = [](uint32_t v) { return (v & 0x7f80u) != 0x7f80u ? 0u : (v & 0x7fu) ? 4u : v >> 15 ? 2u : 1u; };
  return kind(w & 0xffffu) | kind(w >> 16) << 4;
}
__device__ __forceinline__ float marked(float o, uint32_t m) {
  if (m & 1u) o += INFINITY;
  if (m & 2u) o += -INFINITY;
  return m & 4u ? __uint_as_float(0x7fc00000u) : o;
}

// x / group for x below group + kRows + 32 (group_inv: 2^22 / group, rounded up: exact for x < 512)
__device__ __forceinline__ int near_div(const KvAttendDev& at, int x) {
  return at.group >= 256 ? (x >= at.group ? 1 : 0) : (int)(((uint32_t)x * at.group_inv) >> 22);
}

// a lane's maximum of a step's scores (NaN where there is one)
__device__ __forceinline__ float max_of(const f32x16 (&s)[2]) {
  float a = s[0][0], b = s[1][0];
#pragma unroll
  for (int i = 1; i < 15; i += 2) {
    a = __builtin_elementwise_maximum(a, __builtin_elementwise_maximum(s[0][i], s[0][i + 1]));
    b = __builtin_elementwise_maximum(b, __builtin_elementwise_maximum(s[1][i], s[1][i + 1]));
    asm("" : "+v"(a), "+v"(b));
  }
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, s[0][15]), __builtin_elementwise_maximum(b, s[1][15]));
}

// The pipelined step of rows_step (tdk_tiles.h), with the maxima kept in their slots: the scores of the next step's K tile, this step's weights, and the
// products of this step's V tile.  m2: what goes to the scaled scores; mx: each lane's maximum of the new ones.
__device__ __forceinline__ void step_of_rows(const unsigned char* Ks, const unsigned char* Vs, const bf16x8 (&qf)[8], f32x16 (&s)[2], f32x16 (&nx)[2],
                                             float& mx, float scale2, float m2, int lane, RowState& st) {
  constexpr int kAhead = 4, kWeights = 32, kPre = 4;
  const int n = lane & 31, hh = lane >> 5;
  const auto k_op = [&](int j) __attribute__((always_inline)) { return k_operand(Ks + (j & 1) * (kStepTile / 2), j >> 1, n, hh); };
  const auto v_op = [&](int j) __attribute__((always_inline)) { return v_operand(Vs, j >> 2, j & 3, lane); };
  uint32_t pw[4][4];
  // weight number w, in the order the second products need them: 16 tokens at a time; in three stages, each a slot after the one before
  const auto tile = [](int w) { return w / 16; };
  const auto elem = [](int w) { return w % 16; };
  const auto weight = [&](int w) __attribute__((always_inline)) {
    if (w + 2 < kWeights) s[tile(w + 2)][elem(w + 2)] = __builtin_fmaf(s[tile(w + 2)][elem(w + 2)], scale2, m2);
    if (w + 1 < kWeights) s[tile(w + 1)][elem(w + 1)] = __builtin_amdgcn_exp2f(s[tile(w + 1)][elem(w + 1)]);
    st.l_run += s[tile(w)][elem(w)];
    if (w & 1) pw[w / 8][(w % 8) >> 1] = pack2(s[tile(w - 1)][elem(w - 1)], s[tile(w)][elem(w)]);
  };
  __builtin_amdgcn_s_setprio(1);
  bf16x8 ka[kAhead], va[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) ka[j] = k_op(j);
  s[0][0] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][0], scale2, m2));
  s[0][1] = __builtin_fmaf(s[0][1], scale2, m2);
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
    weight(kPre + j);
    __builtin_amdgcn_sched_barrier(0);
  }
  mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[j >> 2][0], pw[j >> 2][1], pw[j >> 2][2], pw[j >> 2][3]});
    st.oacc[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j % kAhead], pb, st.oacc[j & 3], 0, 0, 0);
    if (j + kAhead < 16) va[j % kAhead] = v_op(j + kAhead);
    if (kPre + 16 + j < kWeights) weight(kPre + 16 + j);
    if (j >= 8) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int i = 4 * (j - 8) + 2 * q;
        mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(nx[i >> 4][i & 15], nx[i >> 4][(i & 15) + 1]));
        asm("" : "+v"(mx));                  // (gathered behind the step, as the compiler has it otherwise, they hold up the next)
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
}

// A row's weights are 2^(c (s - m) - 12), s its scores, c the scale times log2 e, m a reference point that follows their maximum only from 2^11.5 on, so that
// sums and products (both fp32) are seldom scaled again; weights go to the second products as bf16 (half a step of 2^-8 each, the error that is left).
// What bounds it: the clock that matrix and vector units share under load.  A prompt of 8192 tokens, 8 heads with 5 queries each: 613 to 659 us by card, 1043 to 1121
// TFLOP/s of what the queries see where a matrix product of 16 384 reaches 1364; counters: matrix cores 65 % busy, vector units 55 %, 1.7 GHz, no bank conflicts.
// Why so: two workgroups of four wavefronts on a compute unit, 32 rows a wavefront.  64 rows a wavefront spill (1175 us for 720 at the time), eight
// wavefronts a workgroup wait for one another (676 for 660, 25 short prompts 158 for 138).  Steps that every row sees whole skip all tests by
// one scalar; the maxima of the next scores stand in the slots of the second products (719 -> 663 us with scalar borders, 655 with that scalar).
// Tried without gain: sums by dot products (689 for 680) or by a product with ones (640 for 610), no raised priority (628 for 610), loads in the
// slots, operands three or six ahead.  Of a short prompt's workgroup (14 us) half is start and end: starts 0.9, tiles 2.6, first scores 1.4.
template <class Source>
__device__ __forceinline__ void attend_in_steps(const KvDev kv, const typename Source::At at) {
  __shared__ __align__(16) StepTiles sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hh = lane >> 5;
  int h;
  const int rest = rest_of<false>(kv.heads, h), chunk = rest % at.n_chunks;
  if (rest >= at.n_rest) return;
  Block b;
  Source src;
  const int place = rest / at.n_chunks;
  if (!src.find(kv, at, place, lane, b)) return;
  h = (h + (src.kSpread ? b.s + chunk : 0)) % kv.heads;
  const int t_begin = (int)min((int64_t)chunk * at.piece_tiles, (int64_t)src.total);
  const int t_end = chunk == at.n_chunks - 1 ? src.total : min(t_begin + at.piece_tiles, src.total);
  if (t_begin == t_end && at.n_chunks > 1) {
    put_empty(at, b, h, chunk, kRows);
    return;
  }

  // the wavefront's own rows: numbers `first` + 0 .. 31 behind the block's first token
  const int w0 = b.r0 + 32 * wave, t0 = b.r0 / at.group, first = w0 - t0 * at.group;
  const bool active = w0 < b.n_rows;
  const int n_on = min(b.n_rows - w0, 32);   // rows that there are
  const int64_t tok0 = b.q0 + t0;
  const int my_tok = near_div(at, first + n);
  const int pos = n < n_on ? b.pos0 + t0 + my_tok : -1;
  const int p_lo = __builtin_amdgcn_readfirstlane(b.pos0 + t0 + near_div(at, first));
  const int p_hi = __builtin_amdgcn_readfirstlane(b.pos0 + t0 + near_div(at, first + max(n_on, 1) - 1));
  src.open(kv, at, b, h, t_begin, t_end, sh, lane, wave);
  bf16x8 qf[8];
  {
    const bool on = n < n_on;
    const char* q = at.q + (on ? tok0 + my_tok : b.q0) * at.q_stride + (on ? h * at.group + first + n - my_tok * at.group : 0) * kRow;
    u32x4 x[8];                              // (rows that there are not: as the block's first, and not written)
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) x[kk] = *reinterpret_cast<const u32x4*>(q + 32 * kk + 16 * hh);
    if (at.q_flip) {
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[kk][e] ^= 0x80008000u;
    }
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = __builtin_bit_cast(bf16x8, x[kk]);
  }
  RowState st;
  row_state_init(st);

  // Scores of what the rows do not see.  Element k of a lane is token 32 (k / 16) + 8 ((k % 16) / 4) + 4 hh + k % 4 of the step.
  const auto token = [](int k) { return 32 * (k >> 4) + 8 * ((k & 15) >> 2) + (k & 3); };
  // Each kind of border in a pass of its own, for the few steps that meet it.
  const auto mask_scores = [&](int j0, int ok, f32x16 (&s)[2], float& mx) __attribute__((always_inline)) {
    const int j1 = j0 + kStep - 1, a = pos - j0 - 4 * hh;
    if (j1 > p_lo) {
#pragma unroll
      for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] = token(k) <= a ? s[k >> 4][k & 15] : -INFINITY;
    }
    if (at.window && p_hi - j0 >= at.window && j1 >= at.n_sink) {
      const int low = (int)((unsigned)a - (unsigned)at.window), sink = at.n_sink - j0 - 4 * hh;
#pragma unroll
      for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] = token(k) > low || token(k) < sink ? s[k >> 4][k & 15] : -INFINITY;
    }
    if (Source::kHoles && (ok != 15 || (j1 >= b.hole_b && j0 < b.hole_e))) {
      const int hb = b.hole_b - j0 - 4 * hh, he = b.hole_e - j0 - 4 * hh;
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        const int t = token(k);
        s[k >> 4][k & 15] = !(t >= hb && t < he) && (ok >> (t >> 4) & 1) ? s[k >> 4][k & 15] : -INFINITY;
      }
    }
    mx = max_of(s);
  };
  constexpr float kFar = 4096.f;             // (as in attend_steps: reference points beyond are subtracted before scaling)
  bool far = false, marks = false;
  const auto settle = [&](float mx) __attribute__((always_inline)) {
    if (!__any(moved(st.m_run, mx, at.scale2) != st.m_run)) return;
    const float m_new = moved(st.m_run, pair_max(mx), at.scale2);
    const float alpha = share(st.m_run, reference(m_new), at.scale2);      // 1 for the rows whose reference point stays
    st.l_run *= alpha;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.oacc[q][i] *= alpha;
    st.m_run = m_new;
    far = __any(fabsf(reference(m_new)) * at.scale2 > kFar);
  };
  if (t_begin < t_end) {
    f32x16 s0[2], s1[2];
    src.first();
    bool whole = src.whole(t_begin, 0);         // every row sees all of this step, and no page is missing
    __syncthreads();
    if (active) {
      float mx;
      rows_scores(sh.k[1], qf, n, hh, s0);
      if (whole) mx = max_of(s0);
      else mask_scores(src.token(t_begin), src.ok(0), s0, mx);
      const float m = pair_max(mx);
      st.m_run = m > -INFINITY ? m : -INFINITY;        // (a NaN: as if there were no score yet)
      far = __any(fabsf(reference(st.m_run)) * at.scale2 > kFar);
    }
    __syncthreads();                         // the first step replaces its K tile
    int i = t_begin;
    // s: this step's scores, nx: the next one's
    const auto step = [&](int place, f32x16 (&s)[2], f32x16 (&nx)[2]) __attribute__((always_inline)) {
      if (!whole) {
        const int flags = sh.odd[place][0] | sh.odd[place][1] | sh.odd[place][2] | sh.odd[place][3];
        if (__builtin_amdgcn_readfirstlane(flags)) {
          // The rows that see what is not finite are marked, and the step meets the rest.  (Rare, so small rather than fast, and apart from the
          // registers of the step.)
          if (!marks) {
            for (int r = 0; r < 32; ++r) sh.marks[32 * wave + r][lane] = 0;
          }
          const int j0 = src.token(i);
#pragma clang loop unroll(disable)
          for (int t = 0; t < kStep; ++t) {
            const uint32_t kinds = odd_kinds(*reinterpret_cast<const uint32_t*>(sh.v[place] + v_place(t, lane >> 2) + 4 * (lane & 3)));
            if (!__any(kinds != 0)) continue;
#pragma clang loop unroll(disable)
            for (int r = 0; r < n_on; ++r)
              if (sees(at, b, b.pos0 + t0 + near_div(at, first + r), j0 + t)) sh.marks[32 * wave + r][lane] |= kinds;
          }
          marks = true;
          __syncthreads();
          u32x4* own = reinterpret_cast<u32x4*>(sh.v[place] + 16 * threadIdx.x);
#pragma unroll
          for (int e = 0; e < 4; ++e) own[256 * e] = kind_of(own[256 * e], 0);
          __syncthreads();
        }
      }
      const bool more = i + 1 < t_end;
      const int ok = src.ok(1);
      whole = more && src.whole(i + 1, 1);
      // (the tiles that are replaced were used up before the last barrier)
      const bool brings = more || !Source::kEnds;
      if (brings) src.bring(i, place ^ 1, more && !whole);
      if (active) {
        if (far) {
          const float ref = reference(st.m_run);
#pragma unroll
          for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] -= ref;
        }
        float mx;
        step_of_rows(sh.k[place], sh.v[place], qf, s, nx, mx, at.scale2, far ? -kBelow : -reference(st.m_run) * at.scale2 - kBelow, lane, st);
        if (!whole) {
          if (more) mask_scores(src.token(i + 1), ok, nx, mx);
          else mx = -INFINITY;               // (past the last step: scores that are not used)
        }
        settle(mx);
      }
      if (brings) {
        src.arrived(i, place ^ 1, more && !whole);
        __syncthreads();
      }
      ++i;
    };
    while (i < t_end) {
      step(0, s0, s1);
      if (i < t_end) step(1, s1, s0);
    }
  }
  if (!active) return;

  // A row's two lanes hold it by four elements in turn.
  float l = st.l_run;
  l += __shfl_xor(l, 32);
  const int own = (int)(threadIdx.x & 31), half = (int)(threadIdx.x >> 5 & 1);       // (n and hh, worked out again rather than kept)
  if (own >= n_on) return;
  const int x = first + own, t = near_div(at, x), hq = h * at.group + x - t * at.group;
  const int64_t row = (tok0 + t) * at.n_q_heads + hq;
  f32x16 (&o)[4] = st.oacc;
  if (marks) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t mk = sh.marks[32 * wave + own][16 * e + 4 * (i >> 2) + 2 * half + ((i & 3) >> 1)];
        o[e][i] = marked(o[e][i], i & 1 ? mk >> 4 : mk & 15u);
      }
  }
  const auto four = [&](int e, int q4) __attribute__((always_inline)) { return f32x4{o[e][4 * q4], o[e][4 * q4 + 1], o[e][4 * q4 + 2], o[e][4 * q4 + 3]}; };
  if (at.n_chunks > 1) {
    const int64_t part = row * at.n_chunks + chunk;
    float* dst = at.part_o + part * kHeadDim + 4 * half;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) *reinterpret_cast<f32x4*>(dst + 32 * e + 8 * q4) = four(e, q4);
    if (half == 0) *reinterpret_cast<f32x2*>(at.part_ml + 2 * part) = f32x2{part_max(st.m_run, l), l};
    return;
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[e][i] *= inv;
  float lse = l > 0.f ? st.m_run * at.scale + __logf(l * kRaise) : l != l ? l : -INFINITY;
  if (at.other_out) {                        // (as in `finish`, all of the row at once)
    const float pl = at.other_lse[row];
    if (pl != -INFINITY) {
      const float* src = at.other_out + row * kHeadDim + 4 * half;
      f32x4 po[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) po[k] = *reinterpret_cast<const f32x4*>(src + 8 * k);
      const float top = fmaxf(lse, pl);
      const float w = lse == top ? 1.f : __expf(lse - top), pw = pl == top ? 1.f : __expf(pl - top), both = w + pw, wb = w / both, pb = pw / both;
#pragma unroll
      for (int k = 0; k < 64; ++k) o[k >> 4][k & 15] = wb * o[k >> 4][k & 15] + pb * po[k >> 2][k & 3];
      lse = top + __logf(both);
    }
  }
  if (at.lse && half == 0) at.lse[row] = lse;
  if (Source::wide(at)) {
    float* dst = reinterpret_cast<float*>(at.out + (tok0 + t) * at.out_stride + hq * (2 * kRow)) + 4 * half;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) *reinterpret_cast<f32x4*>(dst + 32 * e + 8 * q4) = four(e, q4);
    return;
  }
  char* dst = at.out + (tok0 + t) * at.out_stride + hq * kRow + 16 * half;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int q4 = 0; q4 < 4; q4 += 2) {
      // Their halves of the pieces q4 and q4 + 1 (16 bytes of bf16) exchanged: one lane has the one piece, the other the other.
      const f32x4 y = four(e, q4), z = four(e, q4 + 1);
      const auto a = __builtin_amdgcn_permlane32_swap(pack2(y[0], y[1]), pack2(z[0], z[1]), false, false);
      const auto c = __builtin_amdgcn_permlane32_swap(pack2(y[2], y[3]), pack2(z[2], z[3]), false, false);
      *reinterpret_cast<u32x4*>(dst + 16 * (4 * e + q4)) = u32x4{a[0], c[0], a[1], c[1]};
    }
}

}  // namespace

}  // namespace tdk
