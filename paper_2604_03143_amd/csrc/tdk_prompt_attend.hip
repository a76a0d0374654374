// Attention of whole prompts whose rows are not in pages: packed sequences, K and V straight from the projections.
#include "tdk_kv_pages.h"

namespace tdk {

namespace {

constexpr int kStep = kBigTile;              // tokens of a step

// Four wavefronts of 32 NR query rows.
template <int NR>
struct PromptShared {
  unsigned char k[2][kStepTile];
  unsigned char v[2][kStepTile];
  int odd[2][4];                             // per V tile and wavefront: it holds infinity or NaN that only some rows may meet
  uint8_t marks[4 * 32 * NR][kHeadDim / 2];      // of that, what each row has met, by element (four bits each): bit 0 +infinity, 1 -infinity, 2 NaN
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
  // rows 0 .. 63 from `tile` on; those behind `last` repeat that one
  __device__ __forceinline__ void load(const char* tile, int last, uint32_t lds) const {
    if (last >= kStep - 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) load_to_lds(tile + (size_t)(16 * e) * stride, off, lds + 4096u * e + lds_wave);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) load_to_lds(tile, off - (uint32_t)tok * stride + (uint32_t)min(16 * e + tok, last) * stride, lds + 4096u * e + lds_wave);
    }
  }
};

// The block of query rows with this number, as find_block; keys are rows k0 .. k0 + n_keys - 1, the queries belong to the last ones.
__device__ __forceinline__ bool find_rows(const KvDev& kv, const PromptAttendDev& at, int id, int block_rows, int lane, Block& b, int& k0, int& n_keys) {
  int64_t r0 = 0;
  if (id < kv.n_seqs) {
    b.s = id;
  } else {
    const int e = id - kv.n_seqs;
    b.s = count_up_to([&](int i) { return (int64_t)start_of(kv, i) * at.group / block_rows; }, kv.n_seqs, e, lane) - 1;
    if (b.s < 0) return false;
    r0 = (e - (int64_t)start_of(kv, b.s) * at.group / block_rows + 1) * block_rows;
  }
  const int q0 = scalar_read(kv.q_start + b.s), q1 = scalar_read(kv.q_start + b.s + 1);
  const int s0 = scalar_read(at.k_start + b.s), s1 = scalar_read(at.k_start + b.s + 1);
  b.q0 = min(max(q0, 0), kv.n_tokens);
  const int n = min(max(q1, 0), kv.n_tokens) - b.q0;
  k0 = min(max(s0, 0), at.n_k);
  n_keys = max(min(max(s1, 0), at.n_k) - k0, 0);
  b.n_rows = n * at.group;
  if (n <= 0 || r0 >= b.n_rows) return false;
  b.r0 = (int)r0;
  b.pos0 = n_keys - n;                       // (negative: the first queries see nothing)
  b.p_lo = b.pos0 + b.r0 / at.group;
  b.p_hi = b.pos0 + (min(b.r0 + block_rows, b.n_rows) - 1) / at.group;
  b.hole_b = b.hole_e = 0;
  return true;
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

// The pipelined step of tdk_tiles.h for NR tiles of 32 query rows per wavefront: an operand that comes out of LDS meets NR of them.
template <int NR, class Reference>
__device__ __forceinline__ void prompt_step(const unsigned char* Ks, const unsigned char* Vs, const bf16x8 (&qf)[NR][8], f32x16 (&s)[NR][2],
                                            f32x16 (&nx)[NR][2], float (&mx)[NR], float scale2, int lane, RowState (&st)[NR], Reference reference) {
  constexpr int kAhead = 4;
  const int n = lane & 31, hh = lane >> 5;
  float m2[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) m2[r] = reference(r);
  const auto k_op = [&](int j) __attribute__((always_inline)) { return k_operand(Ks + (j & 1) * (kStepTile / 2), j >> 1, n, hh); };
  const auto v_op = [&](int j) __attribute__((always_inline)) { return v_operand(Vs, j >> 2, j & 3, lane); };
  constexpr int kWeights = 32 * NR;
  // weight number w, in the order the second products need them: 16 tokens of every row tile at a time
  uint32_t pw[NR][4][4];
  const auto row = [](int w) { return (w / 8) % NR; };
  const auto tile = [](int w) { return w / (16 * NR); };
  const auto elem = [](int w) { return 8 * ((w / (8 * NR)) & 1) + w % 8; };
  const auto weight = [&](int w) __attribute__((always_inline)) {
    constexpr int a = 2 * NR, c = NR;        // in three stages, each a slot after the one before
    if (w + a < kWeights) s[row(w + a)][tile(w + a)][elem(w + a)] = __builtin_fmaf(s[row(w + a)][tile(w + a)][elem(w + a)], scale2, m2[row(w + a)]);
    if (w + c < kWeights) s[row(w + c)][tile(w + c)][elem(w + c)] = __builtin_amdgcn_exp2f(s[row(w + c)][tile(w + c)][elem(w + c)]);
    const float x = s[row(w)][tile(w)][elem(w)];
    st[row(w)].l_run += x;
    if (w & 1) pw[row(w)][w / (8 * NR)][(w % 8) >> 1] = pack2(s[row(w - 1)][tile(w - 1)][elem(w - 1)], x);
  };
  constexpr int kPre = 4 * NR, kSlot = NR;
  __builtin_amdgcn_s_setprio(1);
  bf16x8 ka[kAhead], va[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) ka[j] = k_op(j);
#pragma unroll
  for (int w = 0; w < 2 * NR; ++w) {
    const float x = __builtin_fmaf(s[row(w)][tile(w)][elem(w)], scale2, m2[row(w)]);
    s[row(w)][tile(w)][elem(w)] = w < NR ? __builtin_amdgcn_exp2f(x) : x;
  }
#pragma unroll
  for (int w = 0; w < kPre; ++w) weight(w);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      f32x16 c;
      if (j < 2) {
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = 0.f;
      } else {
        c = nx[r][j & 1];
      }
      nx[r][j & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[j % kAhead], qf[r][j >> 1], c, 0, 0, 0);
    }
    if (j + kAhead < 16) ka[j % kAhead] = k_op(j + kAhead);
    else va[j % kAhead] = v_op(j + kAhead - 16);
#pragma unroll
    for (int w = 0; w < kSlot; ++w)
      if (kPre + kSlot * j + w < kWeights) weight(kPre + kSlot * j + w);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int r = 0; r < NR; ++r) mx[r] = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pw[r][j >> 2][0], pw[r][j >> 2][1], pw[r][j >> 2][2], pw[r][j >> 2][3]});
      st[r].oacc[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[j % kAhead], pb, st[r].oacc[j & 3], 0, 0, 0);
    }
    if (j + kAhead < 16) va[j % kAhead] = v_op(j + kAhead);
#pragma unroll
    for (int w = 0; w < kSlot; ++w)
      if (kPre + 16 * kSlot + kSlot * j + w < kWeights) weight(kPre + 16 * kSlot + kSlot * j + w);
    if constexpr (NR > 1) {
      if (j >= 4 && j < 8) asm("" : "+v"(nx[(j >> 1) & 1][j & 1]));
    }
    if (j >= 8) {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int i = 4 * (j - 8) + 2 * q;
          mx[r] = __builtin_elementwise_maximum(mx[r], __builtin_elementwise_maximum(nx[r][i >> 4][i & 15], nx[r][i >> 4][(i & 15) + 1]));
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
}

template <int NR>
__device__ __forceinline__ void prompt_attend(const KvDev kv, const PromptAttendDev at) {
  constexpr int kWaveRows = 32 * NR, kRows = 4 * kWaveRows;
  __shared__ __align__(16) PromptShared<NR> sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hh = lane >> 5;
  int h;
  const int rest = rest_of<false>(kv.heads, h), chunk = rest % at.n_chunks;
  if (rest >= at.n_rest) return;
  Block b;
  int k0, n_keys;
  const int place = rest / at.n_chunks;
  if (!find_rows(kv, at, at.last_id < 0 ? place : at.last_id - place, kRows, lane, b, k0, n_keys)) return;
  h = (h + b.s + chunk) % kv.heads;
  const Steps steps = steps_of(at, b);
  const int t_begin = (int)min((int64_t)chunk * at.piece_tiles, (int64_t)steps.total);
  const int t_end = chunk == at.n_chunks - 1 ? steps.total : min(t_begin + at.piece_tiles, steps.total);
  if (t_begin == t_end && at.n_chunks > 1) {
    put_empty(at, b, h, chunk, kRows);
    return;
  }

  // the wavefront's own rows
  const int w0 = b.r0 + kWaveRows * wave;
  const bool active = NR > 1 || w0 < b.n_rows;
  bf16x8 qf[NR][8];
  int pos[NR];
  int p_lo[NR], p_hi[NR];                    // first and last position of each tile's rows
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    const int r = w0 + 32 * rt + n;
    const bool on = r < b.n_rows;
    p_lo[rt] = b.pos0 + min(w0 + 32 * rt, b.n_rows - 1) / at.group;
    p_hi[rt] = b.pos0 + min(w0 + 32 * rt + 31, b.n_rows - 1) / at.group;
    pos[rt] = on ? b.pos0 + r / at.group : -1;
    const int rr = on ? r : b.r0;
    const char* q = at.q + (int64_t)(b.q0 + rr / at.group) * at.q_stride + (h * at.group + rr % at.group) * kRow;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      u32x4 x = *reinterpret_cast<const u32x4*>(q + 32 * kk + 16 * hh);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = on ? (at.q_flip ? x[e] ^ 0x80008000u : x[e]) : 0u;
      qf[rt][kk] = __builtin_bit_cast(bf16x8, x);
    }
  }
  RowState st[NR];
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) row_state_init(st[rt]);
  RowLoader lk, lv;
  lk.template init<false>(at.k_stride);
  lv.template init<true>(at.v_stride);
  const char* const keys = kv.k + (int64_t)k0 * at.k_stride + h * kRow;
  const char* const values = kv.v + (int64_t)k0 * at.v_stride + h * kRow;
  const uint32_t lds_k[2] = {lds_byte(sh.k[0]), lds_byte(sh.k[1])}, lds_v[2] = {lds_byte(sh.v[0]), lds_byte(sh.v[1])};
  // (behind the last step that one is read again: what it gives is not used)
  const auto fetch_k = [&](int i, int buf) __attribute__((always_inline)) {
    const int j0 = steps.token(min(i, t_end - 1));
    lk.load(keys + (int64_t)j0 * at.k_stride, n_keys - 1 - j0, lds_k[buf]);
  };
  const auto fetch_v = [&](int i, int buf) __attribute__((always_inline)) {
    const int j0 = steps.token(min(i, t_end - 1));
    lv.load(values + (int64_t)j0 * at.v_stride, n_keys - 1 - j0, lds_v[buf]);
  };

  // Scores of what the rows do not see.  Bit or element k of a lane is token 32 (k / 16) + 8 ((k % 16) / 4) + 4 hh + k % 4 of the step.
  const auto token = [](int k) { return 32 * (k >> 4) + 8 * ((k & 15) >> 2) + (k & 3); };
  const auto mask_scores = [&](int rt, int j0, f32x16 (&s)[2], float& mx) __attribute__((always_inline)) {
    const int j1 = j0 + kStep - 1;
    const bool late = j1 > p_lo[rt], early = at.window && p_hi[rt] - j0 >= at.window && j1 >= at.n_sink;
    if (!late && !early) return;
    const int a = pos[rt] - j0 - 4 * hh;
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
  const auto settle = [&](float (&mx)[NR]) __attribute__((always_inline)) {
    float m_new[NR];
    bool move = false;
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
      m_new[rt] = moved(st[rt].m_run, pair_max(mx[rt]), at.scale2);
      move |= m_new[rt] != st[rt].m_run;
    }
    if (!__any(move)) return;
    bool f = false;
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
      const float alpha = share(st[rt].m_run, reference(m_new[rt]), at.scale2);      // 1 for the rows whose reference point stays
      st[rt].l_run *= alpha;
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[rt].oacc[q][i] *= alpha;
      st[rt].m_run = m_new[rt];
      f |= fabsf(reference(m_new[rt])) * at.scale2 > kFar;
    }
    far = __any(f);
  };
  // V of a step that some rows see and some do not, before the barrier that hands it over, by the threads that have brought it: what none
  // sees becomes zero (a weight of zero would not silence infinity or NaN), and the tile's flag says whether what is left is finite.
  const auto check_v = [&](int i, int buf) __attribute__((always_inline)) {
    const int j0 = steps.token(i);
    int any = 0;
    if (!all_see(at, b, j0, j0 + kStep - 1)) {
      u32x4* own = reinterpret_cast<u32x4*>(sh.v[buf] + 16 * threadIdx.x);
      bool mine = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u32x4 x = own[256 * e];
        if (!one_sees(at, b, j0 + 16 * e + (int)(threadIdx.x >> 4))) own[256 * e] = u32x4{0, 0, 0, 0};
        else mine |= odd16(x[0]) || odd16(x[1]) || odd16(x[2]) || odd16(x[3]);
      }
      any = __any(mine);
    }
    if (lane == 0) sh.odd[buf][wave] = any;
  };

  if (t_begin < t_end) {
    f32x16 s0[NR][2], s1[NR][2];
    fetch_k(t_begin, 0);
    fetch_v(t_begin, 0);
    fetch_k(t_begin + 1, 1);
    landed();
    check_v(t_begin, 0);
    __syncthreads();
    if (active) {
      float mx[NR];
#pragma unroll
      for (int rt = 0; rt < NR; ++rt) {
        rows_scores(sh.k[0], qf[rt], n, hh, s0[rt]);
        rows_max<2>(s0[rt], mx[rt]);
        mask_scores(rt, steps.token(t_begin), s0[rt], mx[rt]);
      }
      settle(mx);
    }
    __syncthreads();                         // the first step replaces its K tile
    int i = t_begin;
    const auto step = [&](int odd, f32x16 (&s)[NR][2], f32x16 (&nx)[NR][2]) __attribute__((always_inline)) {
      if (sh.odd[odd][0] | sh.odd[odd][1] | sh.odd[odd][2] | sh.odd[odd][3]) {
        // The rows that see what is not finite are marked, and the step meets the rest.  (Rare, so small rather than fast, and apart from the
        // registers of the step.)
        if (!marks) {
          for (int r = 0; r < kWaveRows; ++r) sh.marks[kWaveRows * wave + r][lane] = 0;
        }
        const int j0 = steps.token(i);
#pragma clang loop unroll(disable)
        for (int t = 0; t < kStep; ++t) {
          const uint32_t kinds = odd_kinds(*reinterpret_cast<const uint32_t*>(sh.v[odd] + v_place(t, lane >> 2) + 4 * (lane & 3)));
          if (!__any(kinds != 0)) continue;
#pragma clang loop unroll(disable)
          for (int r = 0; r < kWaveRows && w0 + r < b.n_rows; ++r)
            if (sees(at, b, b.pos0 + (w0 + r) / at.group, j0 + t)) sh.marks[kWaveRows * wave + r][lane] |= kinds;
        }
        marks = true;
        __syncthreads();
        u32x4* own = reinterpret_cast<u32x4*>(sh.v[odd] + 16 * threadIdx.x);
#pragma unroll
        for (int e = 0; e < 4; ++e) own[256 * e] = kind_of(own[256 * e], 0);
        __syncthreads();
      }
      fetch_k(i + 2, odd);
      fetch_v(i + 1, odd ^ 1);
      if (active) {
        // (past the last step: scores that are not used)
        if (far) {
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) {
            const float ref = reference(st[rt].m_run);
#pragma unroll
            for (int k = 0; k < 32; ++k) s[rt][k >> 4][k & 15] -= ref;
          }
        }
        float mx[NR];
        prompt_step<NR>(sh.k[odd ^ 1], sh.v[odd], qf, s, nx, mx, at.scale2, lane, st,
                        [&](int rt) { return far ? -kBelow : -reference(st[rt].m_run) * at.scale2 - kBelow; });
        if (i + 1 < t_end) {
#pragma unroll
          for (int rt = 0; rt < NR; ++rt) mask_scores(rt, steps.token(i + 1), nx[rt], mx[rt]);
          settle(mx);
        }
      }
      landed();
      if (i + 1 < t_end) check_v(i + 1, odd ^ 1);
      __syncthreads();
      ++i;
    };
    while (i < t_end) {
      step(0, s0, s1);
      if (i < t_end) step(1, s1, s0);
    }
  }

  // The rows go out by way of LDS, where 16 lanes hold one: piece c (16 bytes) of row n stands at place c ^ n.
  char* turn = reinterpret_cast<char*>(&sh) + wave * 32 * 4 * kHeadDim;
  static_assert(4 * 32 * 4 * kHeadDim <= sizeof(sh.k) + sizeof(sh.v), "a wavefront's rows lie over the tiles");
  const int piece = lane & 15;
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    float l = st[rt].l_run;
    l += __shfl_xor(l, 32);
    const float m = part_max(st[rt].m_run, l);
    wave_sync();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<f32x4*>(turn + n * 512 + 16 * ((8 * e + 2 * q4 + hh) ^ n)) =
            f32x4{st[rt].oacc[e][4 * q4], st[rt].oacc[e][4 * q4 + 1], st[rt].oacc[e][4 * q4 + 2], st[rt].oacc[e][4 * q4 + 3]};
    wave_sync();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int row = 4 * k + (lane >> 4), rr = w0 + 32 * rt + row;
      const float rm = __shfl(m, row), rl = __shfl(l, row);
      if (rr >= b.n_rows) continue;
      const f32x4 x = *reinterpret_cast<const f32x4*>(turn + row * 512 + 16 * ((2 * piece) ^ row));
      const f32x4 y = *reinterpret_cast<const f32x4*>(turn + row * 512 + 16 * ((2 * piece + 1) ^ row));
      float o[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      if (marks) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t m = sh.marks[kWaveRows * wave + 32 * rt + row][4 * piece + e];
          o[2 * e] = marked(o[2 * e], m & 15u);
          o[2 * e + 1] = marked(o[2 * e + 1], m >> 4);
        }
      }
      put_row(at, b.q0 + rr / at.group, h * at.group + rr % at.group, chunk, piece, o, rm, rl);
    }
  }
}

}  // namespace

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_prompt_attend_kernel(const KvDev kv, const PromptAttendDev at) {
  prompt_attend<1>(kv, at);
}
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void tdk_prompt_attend_wide_kernel(const KvDev kv, const PromptAttendDev at) {
  prompt_attend<2>(kv, at);
}

__global__ __launch_bounds__(256) void tdk_prompt_join_kernel(const KvDev kv, const PromptAttendDev at, int64_t rows) { join_parts(kv, at, rows); }

hipError_t launch_prompt_attend(const KvDev& kv, const PromptAttendDev& at, const KvAttendPlan& p, hipStream_t st) {
  const int64_t blocks = (p.ids * p.n_chunks + 7) / 8 * 8 * kv.heads;
  const hipError_t e = launch(p.block_rows == 256 ? tdk_prompt_attend_wide_kernel : tdk_prompt_attend_kernel, blocks, 256, st, kv, at);
  return e == hipSuccess && p.n_chunks > 1 ? launch(tdk_prompt_join_kernel, (p.rows + 3) / 4, 256, st, kv, at, p.rows) : e;
}

}  // namespace tdk
