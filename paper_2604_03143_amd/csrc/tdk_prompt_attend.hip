// Attention of whole prompts whose rows are not in pages: packed sequences, K and V straight from the projections.  The rows of a block are (token, query
// head of the group) pairs of one sequence and KV head, so that a head's queries share its tiles.  (attend_in_steps has the mathematics and what bounds it.)
// Every (sequence, KV head) stays on one XCD as far as the launch order decides, whose L2 holds its K and V.
#include "tdk_steps.h"

namespace tdk {

namespace {

using u16x2 = uint16_t __attribute__((ext_vector_type(2)));

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
      // load_to_lds four times: the wait states for the addresses once, one for M0 each (8192 tokens, 5 queries a head: 610 -> 605 us)
      asm volatile(
          "s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
          "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
          "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %4\n\t"
          "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5"
          :
          : "s"(lds + lds_wave), "v"(off), "s"(tile), "s"(tile + (size_t)16 * stride), "s"(tile + (size_t)32 * stride), "s"(tile + (size_t)48 * stride)
          : "memory", "scc");
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
  if (n <= 0 || (uint64_t)r0 >= (uint64_t)b.n_rows) return false;       // (negative where the starts decrease)
  b.r0 = (int)r0;
  b.pos0 = n_keys - n;                       // (negative: the first queries see nothing)
  b.p_lo = b.pos0 + b.r0 / at.group;
  b.p_hi = b.pos0 + (min(b.r0 + kRows, b.n_rows) - 1) / at.group;
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

// Rows from memory straight into LDS.
struct RowSource {
  using At = PromptAttendDev;
  static constexpr bool kHoles = false, kSpread = true, kEnds = true;       // (25 prompts of 300 tokens 70 -> 66 us)
  static __device__ __forceinline__ bool wide(const At& at) { return at.f32; }

  int k0, n_keys, total;
  Steps steps;
  __device__ __forceinline__ bool find(const KvDev& kv, const At& at, int place, int lane, Block& b) {
    if (!find_rows(kv, at, place < at.down ? at.last_id - place : place - at.down, lane, b, k0, n_keys)) return false;
    steps = steps_of(at, b);
    total = steps.total;
    return true;
  }

  const At* a;
  const Block* blk;
  StepTiles* sh;
  RowLoader lk, lv;
  const char *keys, *values;
  uint32_t lds_k, lds_v;
  int t_begin, t_end, rows, wave, lane;
  __device__ __forceinline__ void open(const KvDev& kv, const At& at, const Block& b, int h, int begin, int end, StepTiles& tiles, int lane_, int wave_) {
    a = &at;
    blk = &b;
    sh = &tiles;
    lane = lane_;
    wave = wave_;
    t_begin = begin;
    t_end = end;
    lk.init<false>(at.k_stride);
    lv.init<true>(at.v_stride);
    keys = kv.k + (int64_t)k0 * at.k_stride + h * kRow;
    values = kv.v + (int64_t)k0 * at.v_stride + h * kRow;
    lds_k = lds_byte(tiles.k[0]);
    lds_v = lds_byte(tiles.v[0]);
    rows = at.n_k - k0;
    if (begin < end) {
      fetch_k(begin, 1);
      fetch_v(begin, 0);
      if (begin + 1 < end) fetch_k(begin + 1, 0);
    }
  }
  __device__ __forceinline__ int token(int i) const { return steps.token(i); }
  __device__ __forceinline__ int ok(int) const { return 15; }
  __device__ __forceinline__ bool whole(int i, int) const {
    const int j0 = steps.token(i);
    return (j0 + kStep - 1 <= blk->p_lo) & ((a->window == 0) | (blk->p_hi - j0 < a->window));
  }
  // (Rows behind the sequence's are read as they come, up to the end of the buffer, and not seen.)
  __device__ __forceinline__ void fetch_k(int i, int place) const {
    const int j0 = steps.token(i);
    lk.load(keys + (int64_t)j0 * a->k_stride, rows - j0, lds_k + (uint32_t)place * kStepTile);
  }
  __device__ __forceinline__ void fetch_v(int i, int place) const {
    const int j0 = steps.token(i);
    lv.load(values + (int64_t)j0 * a->v_stride, rows - j0, lds_v + (uint32_t)place * kStepTile);
  }
  // V of a step that some rows see and some do not, before the barrier that hands it over, by the threads that have brought it: what none
  // sees becomes zero (a weight of zero would not silence infinity or NaN), and the tile's flag says whether what is left is finite.
  __device__ __forceinline__ void check_v(int i, int place) const {
    const int j0 = steps.token(i);
    u32x4* own = reinterpret_cast<u32x4*>(sh->v[place] + 16 * threadIdx.x);
    u32x4 x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = own[256 * e];
    u16x2 top = {0, 0};                      // the largest magnitudes, as bits: infinity and NaN are above all that is finite
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = j0 + 16 * e + (int)(threadIdx.x >> 4);
      const bool seen = (j <= blk->p_hi) & ((a->window == 0) | (blk->p_lo - j < a->window) | (j < a->n_sink));
      const uint32_t size = seen ? 0x7fff7fffu : 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[e][k] & size));
      if (!seen) own[256 * e] = u32x4{0, 0, 0, 0};
    }
    const int any = __any(max((int)top[0], (int)top[1]) >= 0x7f80);
    if (lane == 0) sh->odd[place][wave] = any;
  }
  __device__ __forceinline__ void first() const {
    landed();
    // The queries are there by now too, and the compiler has to see it: else it waits for their registers in the loop, and so for the tiles on their way.
    __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    if (!whole(t_begin, 0)) check_v(t_begin, 0);
  }
  __device__ __forceinline__ void bring(int i, int place, bool) const {
    if (i + 2 < t_end) fetch_k(i + 2, place);
    fetch_v(i + 1, place);
  }
  __device__ __forceinline__ void arrived(int i, int place, bool check) const {
    landed();
    if (check) check_v(i + 1, place);
  }
};

}  // namespace

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_prompt_attend_kernel(const KvDev kv, const PromptAttendDev at) {
  attend_in_steps<RowSource>(kv, at);
}

__global__ __launch_bounds__(256) void tdk_prompt_join_kernel(const KvDev kv, const PromptAttendDev at, int64_t rows) { join_parts(kv, at, rows); }

hipError_t launch_prompt_attend(const KvDev& kv, const PromptAttendDev& at, const KvAttendPlan& p, hipStream_t st) {
  const int64_t blocks = (p.ids * p.n_chunks + 7) / 8 * 8 * kv.heads;
  const hipError_t e = launch(tdk_prompt_attend_kernel, blocks, 256, st, kv, at);
  return e == hipSuccess && p.n_chunks > 1 ? launch(tdk_prompt_join_kernel, (p.rows + 3) / 4, 256, st, kv, at, p.rows) : e;
}

}  // namespace tdk
