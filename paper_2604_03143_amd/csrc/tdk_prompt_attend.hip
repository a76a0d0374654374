// Attention of whole prompts whose rows are not in pages: packed sequences, K and V straight from the projections.
#include "tdk_kv_pages.h"

namespace tdk {

namespace {

constexpr int kStep = kBigTile;              // tokens of a step
constexpr int kRows = 4 * 32;                // query rows of a workgroup, 32 per wavefront

struct PromptShared {
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

// One thread's share of the loads of a step's tile, rows `stride` bytes apart: piece t % 16 of rows t / 16, 16 + t / 16, ...
struct RowLoader {
  uint32_t stride, off;
  int tok;
  uint32_t lds_wave;
  template <bool V>
  __device__ __forceinline__ void init(int64_t row_bytes) {
    stride = (uint32_t)row_bytes;            // (below 2^26: offsets inside a tile fit 32 bits)
    tok = threadIdx.x >> 4;
    off = (uint32_t)tok * stride + 16u * ((threadIdx.x & 15) ^ (V ? 4 * (tok & 3) : tok & 15));
    lds_wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * 1024u;
  }
  // a tile of `rows` rows up to the end of the buffer: those behind repeat the last
  __device__ __forceinline__ void load(const char* tile, int rows, uint32_t lds) const {
    if (rows >= kStep) {
#pragma unroll
      for (int e = 0; e < 4; ++e) load_to_lds(tile + (size_t)(16 * e) * stride, off, lds + 4096u * e + lds_wave);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) load_to_lds(tile, off - (uint32_t)tok * stride + (uint32_t)min(16 * e + tok, rows - 1) * stride, lds + 4096u * e + lds_wave);
    }
  }
};

// The row block with this number (numbered as in find_block); keys are rows k0 .. k0 + n_keys - 1, the queries belong to the last ones.
__device__ __forceinline__ bool find_rows(const KvDev& kv, const PromptAttendDev& at, int id, int lane, Block& b, int& k0, int& n_keys) {
  int64_t r0 = 0;
  int q1, k1;
  if (kv.n_seqs < 64) {                      // all starts in one read
    const int i = min(lane, kv.n_seqs);
    const int q = min(max(kv.q_start[i], 0), kv.n_tokens), k = min(max(at.k_start[i], 0), at.n_k);
    if (id < kv.n_seqs) {
      b.s = id;
    } else {
      const int e = id - kv.n_seqs;
      b.s = __popcll(__ballot(lane < kv.n_seqs && (int64_t)q * at.group / kRows <= e)) - 1;
      if (b.s < 0) return false;
      r0 = (e - (int64_t)__builtin_amdgcn_readlane(q, b.s) * at.group / kRows + 1) * kRows;
    }
    b.q0 = __builtin_amdgcn_readlane(q, b.s);
    q1 = __builtin_amdgcn_readlane(q, b.s + 1);
    k0 = __builtin_amdgcn_readlane(k, b.s);
    k1 = __builtin_amdgcn_readlane(k, b.s + 1);
  } else {
    if (id < kv.n_seqs) {
      b.s = id;
    } else {
      const int e = id - kv.n_seqs;
      b.s = count_up_to([&](int i) { return (int64_t)start_of(kv, i) * at.group / kRows; }, kv.n_seqs, e, lane) - 1;
      if (b.s < 0) return false;
      r0 = (e - (int64_t)start_of(kv, b.s) * at.group / kRows + 1) * kRows;
    }
    const int a0 = scalar_read(kv.q_start + b.s), a1 = scalar_read(kv.q_start + b.s + 1);
    const int c0 = scalar_read(at.k_start + b.s), c1 = scalar_read(at.k_start + b.s + 1);
    b.q0 = min(max(a0, 0), kv.n_tokens);
    q1 = min(max(a1, 0), kv.n_tokens);
    k0 = min(max(c0, 0), at.n_k);
    k1 = min(max(c1, 0), at.n_k);
  }
  const int n = q1 - b.q0;
  n_keys = max(k1 - k0, 0);
  b.n_rows = n * at.group;
  if (n <= 0 || r0 < 0 || r0 >= b.n_rows) return false;
  b.r0 = (int)r0;
  b.pos0 = n_keys - n;                       // (negative: the first queries see nothing)
  b.p_lo = b.pos0 + b.r0 / at.group;
  b.p_hi = b.pos0 + (min(b.r0 + kRows, b.n_rows) - 1) / at.group;
  b.hole_b = b.hole_e = 0;
  return true;
}

// x / group for x below group + kRows (group_inv: 2^22 / group, rounded up: exact for x < 512)
__device__ __forceinline__ int near_div(const PromptAttendDev& at, int x) {
  return at.group >= 256 ? (x >= at.group ? 1 : 0) : (int)(((uint32_t)x * at.group_inv) >> 22);
}

// The steps that hold what some row of the block sees: first tokens, then the window.
struct Steps {
  int sink, near, total;                     // steps of the first tokens, first step of the window
  __device__ __forceinline__ int token(int i) const { return kStep * (i < sink ? i : near + i - sink); }
};
__device__ __forceinline__ Steps steps_of(const PromptAttendDev& at, const Block& b) {
  const int end = b.p_hi + 1;                // (at most the keys there are)
  int near = at.window ? (int)max((int64_t)0, (int64_t)b.p_lo - at.window + 1) : 0, sink = at.window ? min(at.n_sink, end) : 0;
  Steps t;
  t.sink = (max(sink, 0) + kStep - 1) / kStep;
  t.near = max(near / kStep, t.sink);
  t.total = t.sink + max(0, (max(end, 0) + kStep - 1) / kStep - t.near);
  return t;
}

// The pipelined step of rows_step (tdk_tiles.h), with the maxima kept in their slots: the scores of the next step's K tile, this step's weights, and the
// products of this step's V tile.  m2: what goes to the scaled scores; mx: each lane's maximum of the new ones.
__device__ __forceinline__ void prompt_step(const unsigned char* Ks, const unsigned char* Vs, const bf16x8 (&qf)[8], f32x16 (&s)[2], f32x16 (&nx)[2],
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

}  // namespace

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_prompt_attend_kernel(const KvDev kv, const PromptAttendDev at) {
  __shared__ __align__(16) PromptShared sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hh = lane >> 5;
  int h;
  const int rest = rest_of<false>(kv.heads, h), chunk = rest % at.n_chunks;
  if (rest >= at.n_rest) return;
  Block b;
  int k0, n_keys;
  const int place = rest / at.n_chunks;
  if (!find_rows(kv, at, place < at.down ? at.last_id - place : place - at.down, lane, b, k0, n_keys)) return;
  h = (h + b.s + chunk) % kv.heads;
  const Steps steps = steps_of(at, b);
  const int t_begin = (int)min((int64_t)chunk * at.piece_tiles, (int64_t)steps.total);
  const int t_end = chunk == at.n_chunks - 1 ? steps.total : min(t_begin + at.piece_tiles, steps.total);
  if (t_begin == t_end && at.n_chunks > 1) {
    put_empty(at, b, h, chunk, kRows);
    return;
  }

  // the wavefront's own rows: numbers `first` + 0 .. 31 behind the block's first token
  const int w0 = b.r0 + 32 * wave, t0 = b.r0 / at.group, first = w0 - t0 * at.group;
  const bool active = w0 < b.n_rows;
  const int n_on = min(b.n_rows - w0, 32);   // rows that there are
  const int64_t tok0 = b.q0 + t0;
  const int my_tok = near_div(at, first + n), my_head = h * at.group + first + n - my_tok * at.group;
  const int pos = n < n_on ? b.pos0 + t0 + my_tok : -1;
  const int p_lo = __builtin_amdgcn_readfirstlane(b.pos0 + t0 + near_div(at, first));
  const int p_hi = __builtin_amdgcn_readfirstlane(b.pos0 + t0 + near_div(at, first + max(n_on, 1) - 1));
  RowLoader lk, lv;
  lk.init<false>(at.k_stride);
  lv.init<true>(at.v_stride);
  const char* const keys = kv.k + (int64_t)k0 * at.k_stride + h * kRow;
  const char* const values = kv.v + (int64_t)k0 * at.v_stride + h * kRow;
  const uint32_t lds_k = lds_byte(sh.k[0]), lds_v = lds_byte(sh.v[0]);
  // (Behind the last step that one is read again: what it gives is not used.  Rows behind the sequence's are read as they come, up to the end of the buffer,
  // and not seen.)
  const int rows = at.n_k - k0;
  const auto fetch_k = [&](int i, int buf) __attribute__((always_inline)) {
    const int j0 = steps.token(min(i, t_end - 1));
    lk.load(keys + (int64_t)j0 * at.k_stride, rows - j0, lds_k + (uint32_t)buf * kStepTile);
  };
  const auto fetch_v = [&](int i, int buf) __attribute__((always_inline)) {
    const int j0 = steps.token(min(i, t_end - 1));
    lv.load(values + (int64_t)j0 * at.v_stride, rows - j0, lds_v + (uint32_t)buf * kStepTile);
  };
  // V tile j and K tile j + 1 (counted from the part's first step) lie in place j % 2.
  if (t_begin < t_end) {
    fetch_k(t_begin, 1);
    fetch_v(t_begin, 0);
    fetch_k(t_begin + 1, 0);
  }
  bf16x8 qf[8];
  {
    const bool on = n < n_on;
    const char* q = at.q + (on ? tok0 + my_tok : b.q0) * at.q_stride + (on ? my_head : 0) * kRow;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      u32x4 x = *reinterpret_cast<const u32x4*>(q + 32 * kk + 16 * hh);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = on ? (at.q_flip ? x[e] ^ 0x80008000u : x[e]) : 0u;
      qf[kk] = __builtin_bit_cast(bf16x8, x);
    }
  }
  RowState st;
  row_state_init(st);

  // Scores of what the rows do not see.  Element k of a lane is token 32 (k / 16) + 8 ((k % 16) / 4) + 4 hh + k % 4 of the step.
  const auto token = [](int k) { return 32 * (k >> 4) + 8 * ((k & 15) >> 2) + (k & 3); };
  const auto mask_scores = [&](int j0, f32x16 (&s)[2], float& mx) __attribute__((always_inline)) {
    const int j1 = j0 + kStep - 1;
    const bool late = j1 > p_lo, early = at.window && p_hi - j0 >= at.window && j1 >= at.n_sink;
    if (!late && !early) return;
    const int a = pos - j0 - 4 * hh;
    if (late) {
#pragma unroll
      for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] = token(k) <= a ? s[k >> 4][k & 15] : -INFINITY;
    }
    if (early) {
      const int low = (int)((unsigned)a - (unsigned)at.window), sink = at.n_sink - j0 - 4 * hh;
#pragma unroll
      for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] = token(k) > low || token(k) < sink ? s[k >> 4][k & 15] : -INFINITY;
    }
    rows_max<2>(s, mx);
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
  // V of a step that some rows see and some do not, before the barrier that hands it over, by the threads that have brought it: what none
  // sees becomes zero (a weight of zero would not silence infinity or NaN), and the tile's flag says whether what is left is finite.
  const auto check_v = [&](int i, int buf) __attribute__((always_inline)) {
    const int j0 = steps.token(i);
    u32x4* own = reinterpret_cast<u32x4*>(sh.v[buf] + 16 * threadIdx.x);
    bool mine = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const u32x4 x = own[256 * e];
      if (!one_sees(at, b, j0 + 16 * e + (int)(threadIdx.x >> 4))) own[256 * e] = u32x4{0, 0, 0, 0};
      else mine |= odd16(x[0]) || odd16(x[1]) || odd16(x[2]) || odd16(x[3]);
    }
    const int any = __any(mine);
    if (lane == 0) sh.odd[buf][wave] = any;
  };
  // steps that every row of the block sees whole: [seen_from, seen_to)
  const int seen_from = at.window ? steps.sink + max(0, max(b.p_hi - at.window + kStep, 0) / kStep - steps.near) : 0;
  const int seen_to = at.window ? steps.sink + max(0, (max(b.p_lo, -1) + 1) / kStep - steps.near) : (max(b.p_lo, -1) + 1) / kStep;
  const auto seen = [&](int i) { return i >= seen_from && i < seen_to; };

  if (t_begin < t_end) {
    f32x16 s0[2], s1[2];
    landed();
    if (!seen(t_begin)) check_v(t_begin, 0);
    __syncthreads();
    if (active) {
      float mx;
      rows_scores(sh.k[1], qf, n, hh, s0);
      rows_max<2>(s0, mx);
      mask_scores(steps.token(t_begin), s0, mx);
      const float m = pair_max(mx);
      st.m_run = m > -INFINITY ? m : -INFINITY;        // (a NaN: as if there were no score yet)
      far = __any(fabsf(reference(st.m_run)) * at.scale2 > kFar);
    }
    __syncthreads();                         // the first step replaces its K tile
    int i = t_begin;
    // s: this step's scores, nx: the next one's
    const auto step = [&](int place, f32x16 (&s)[2], f32x16 (&nx)[2]) __attribute__((always_inline)) {
      if (!seen(i)) {
        const int flags = sh.odd[place][0] | sh.odd[place][1] | sh.odd[place][2] | sh.odd[place][3];
        if (__builtin_amdgcn_readfirstlane(flags)) {
          // The rows that see what is not finite are marked, and the step meets the rest.  (Rare, so small rather than fast, and apart from the
          // registers of the step.)
          if (!marks) {
            for (int r = 0; r < 32; ++r) sh.marks[32 * wave + r][lane] = 0;
          }
          const int j0 = steps.token(i);
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
      // (the tiles that are replaced were used up before the last barrier)
      fetch_k(i + 2, place ^ 1);
      fetch_v(i + 1, place ^ 1);
      if (active) {
        if (far) {
          const float ref = reference(st.m_run);
#pragma unroll
          for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] -= ref;
        }
        float mx;
        prompt_step(sh.k[place], sh.v[place], qf, s, nx, mx, at.scale2, far ? -kBelow : -reference(st.m_run) * at.scale2 - kBelow, lane, st);
        if (!seen(i + 1)) {
          mask_scores(steps.token(i + 1), nx, mx);
          if (i + 1 >= t_end) mx = -INFINITY;          // (past the last step: scores that are not used)
        }
        settle(mx);
      }
      ++i;
      landed();
      if (!seen(i) && i < t_end) check_v(i, place ^ 1);
      __syncthreads();
    };
    while (i < t_end) {
      step(0, s0, s1);
      if (i < t_end) step(1, s1, s0);
    }
  }
  if (!active) return;

  // The rows go out by way of LDS, where 16 lanes hold one: piece c (16 bytes) of row n stands at place c ^ n.
  float l = st.l_run;
  l += __shfl_xor(l, 32);
  const int piece = lane & 15;
  if (at.n_chunks == 1 && !at.other_out && !at.f32 && !marks) {
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    if (at.lse && hh == 0 && n < n_on) at.lse[(tok0 + my_tok) * at.n_q_heads + my_head] = l > 0.f ? st.m_run * at.scale + __logf(l * kRaise) : l != l ? l : -INFINITY;
    char* turn = reinterpret_cast<char*>(&sh) + wave * 32 * kRow;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<u32x2*>(turn + n * kRow + 16 * ((4 * e + q4) ^ (n & 15)) + 8 * hh) =
            u32x2{pack2(st.oacc[e][4 * q4] * inv, st.oacc[e][4 * q4 + 1] * inv), pack2(st.oacc[e][4 * q4 + 2] * inv, st.oacc[e][4 * q4 + 3] * inv)};
    wave_sync();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int row = 4 * k + (lane >> 4);
      if (row >= n_on) continue;
      const int t = near_div(at, first + row);
      *reinterpret_cast<u32x4*>(at.out + (tok0 + t) * at.out_stride + (h * at.group + first + row - t * at.group) * kRow + 16 * piece) =
          *reinterpret_cast<const u32x4*>(turn + row * kRow + 16 * (piece ^ (row & 15)));
    }
    return;
  }
  char* turn = reinterpret_cast<char*>(&sh) + wave * 32 * 4 * kHeadDim;
  static_assert(4 * 32 * 4 * kHeadDim <= sizeof(sh.k) + sizeof(sh.v), "a wavefront's rows lie over the tiles");
  const float m = part_max(st.m_run, l);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      *reinterpret_cast<f32x4*>(turn + n * 512 + 16 * ((8 * e + 2 * q4 + hh) ^ n)) =
          f32x4{st.oacc[e][4 * q4], st.oacc[e][4 * q4 + 1], st.oacc[e][4 * q4 + 2], st.oacc[e][4 * q4 + 3]};
  wave_sync();
#pragma clang loop unroll(disable)
  for (int k = 0; k < 8; ++k) {
    const int row = 4 * k + (lane >> 4);
    const float rm = __shfl(m, row), rl = __shfl(l, row);
    if (row >= n_on) continue;
    const f32x4 x = *reinterpret_cast<const f32x4*>(turn + row * 512 + 16 * ((2 * piece) ^ row));
    const f32x4 y = *reinterpret_cast<const f32x4*>(turn + row * 512 + 16 * ((2 * piece + 1) ^ row));
    float o[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    if (marks) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t mk = sh.marks[32 * wave + row][4 * piece + e];
        o[2 * e] = marked(o[2 * e], mk & 15u);
        o[2 * e + 1] = marked(o[2 * e + 1], mk >> 4);
      }
    }
    const int t = near_div(at, first + row);
    put_row(at, tok0 + t, h * at.group + first + row - t * at.group, chunk, piece, o, rm, rl);
  }
}

__global__ __launch_bounds__(256) void tdk_prompt_join_kernel(const KvDev kv, const PromptAttendDev at, int64_t rows) { join_parts(kv, at, rows); }

hipError_t launch_prompt_attend(const KvDev& kv, const PromptAttendDev& at, const KvAttendPlan& p, hipStream_t st) {
  const int64_t blocks = (p.ids * p.n_chunks + 7) / 8 * 8 * kv.heads;
  const hipError_t e = launch(tdk_prompt_attend_kernel, blocks, 256, st, kv, at);
  return e == hipSuccess && p.n_chunks > 1 ? launch(tdk_prompt_join_kernel, (p.rows + 3) / 4, 256, st, kv, at, p.rows) : e;
}

}  // namespace tdk
