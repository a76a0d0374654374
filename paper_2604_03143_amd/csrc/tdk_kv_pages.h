// Caches that programs append to: new tokens into the pages (rotated on the way, in bf16, in 8 bits or in 4), attention of their
// queries to the pages, and rows back out of them.  The kernels' bodies by the format of the pages: the files that include this give them their names.
#pragma once

#include "tdk_kv.h"
#include "tdk_internal.h"
#include "tdk_tiles.h"

#include <type_traits>

namespace tdk {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int kRow = 2 * kHeadDim;         // bytes of a bf16 head row
constexpr int kRow4 = kHeadDim / 2;        // bytes of its 4-bit values
constexpr int kRow8 = kHeadDim;            // bytes of its 8-bit values

constexpr int code_bytes(int fmt) { return fmt == kMx4 ? kRow4 : kRow8; }      // bytes of a head row's values; four of exponents come behind a page's

// Accesses that pass the caches by, for what is met once.
template <class T>
__device__ __forceinline__ T load_once(const char* p) { return __builtin_nontemporal_load(reinterpret_cast<const T*>(p)); }
template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const char* p) {
  return ONCE ? load_once<u32x4>(p) : *reinterpret_cast<const u32x4*>(p);
}
template <bool ONCE>
__device__ __forceinline__ void store16(char* p, u32x4 v) {
  if (ONCE) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
  else *reinterpret_cast<u32x4*>(p) = v;
}

// For i in [0, n), at(i) not decreasing: how many are <= x.  The lanes of a wavefront probe 64 places a round (one round up to
// 64 entries, two up to 4096).  A round leaves less than a 64th of the range, whatever the values are.
template <class F>
__device__ __forceinline__ int count_up_to(F at, int n, int64_t x, int lane) {
  int lo = 0, hi = n;
  while (hi > lo) {
    const int step = (hi - lo + 63) / 64;
    const int64_t i = lo + (int64_t)step * (lane + 1) - 1;
    const bool le = i < hi && at((int)i) <= x;
    const int c = __popcll(__ballot(le));
    const int64_t next = lo + (int64_t)step * c, last = lo + (int64_t)step * (c + 1) - 1;
    lo = (int)min((int64_t)hi, next);
    hi = (int)max((int64_t)lo, min((int64_t)hi, last));
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A start out of q_start, cut to the token buffers.
__device__ __forceinline__ int start_of(const KvDev& kv, int i) { return min(max(kv.q_start[i], 0), kv.n_tokens); }

// Physical page of a sequence's logical page, -1 where there is none.
__device__ __forceinline__ int page_of(const KvDev& kv, int s, int64_t lp) {
  if (lp < 0 || lp >= kv.table_stride) return -1;
  const int p = kv.table[(int64_t)s * kv.table_stride + lp];
  return p >= 0 && p < kv.pool_pages ? p : -1;
}

// Where a row of the token buffers belongs: -1 for rows that no sequence has or whose place the table does not name.
struct Slot { int page, at, pos; };
__device__ __forceinline__ Slot slot_of(const KvDev& kv, int row, int lane) {
  const int s = count_up_to([&](int i) { return (int64_t)start_of(kv, i + 1); }, kv.n_seqs, row, lane);
  Slot o{-1, 0, -1};
  if (s >= kv.n_seqs) return o;
  const int q0 = start_of(kv, s), q1 = start_of(kv, s + 1);
  if (row < q0 || row >= q1) return o;
  const int pos = max(kv.seq_len[s], 0) - (q1 - row);
  if (pos < 0) return o;
  o.page = page_of(kv, s, pos >> kv.page_shift);
  o.at = pos & ((1 << kv.page_shift) - 1);
  o.pos = pos;
  return o;
}

// The values of a head row in a 4-bit or 8-bit page, and its four block exponents.
template <int FMT>
__device__ __forceinline__ char* code_row(char* plane, const KvDev& kv, const Slot& o, int h) {
  const int T = 1 << kv.page_shift;
  return plane + ((int64_t)o.page * kv.heads + h) * (T * (code_bytes(FMT) + 4)) + o.at * code_bytes(FMT);
}
template <int FMT>
__device__ __forceinline__ char* code_scales(char* plane, const KvDev& kv, const Slot& o, int h) {
  const int T = 1 << kv.page_shift;
  return plane + ((int64_t)o.page * kv.heads + h) * (T * (code_bytes(FMT) + 4)) + T * code_bytes(FMT) + o.at * 4;
}

__device__ __forceinline__ uint32_t top_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  // the block: four lanes of eight elements
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  return max(m, (uint32_t)__shfl_xor((int)m, 2));
}

// The byte of a block's power of two from the bits of its largest magnitude: the exponent, one more where the mantissa is 1.75 or
// above (a carry out of the bits below), less the two of the largest 4-bit value.  Infinities and NaN lie above all numbers.
__device__ __forceinline__ uint32_t block_exponent(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = (int)((top + 0x200000u) >> 23) - 2;
  return (uint32_t)max(e, 1);
}

__device__ __forceinline__ uint32_t to4(const float (&x)[8], uint32_t e) {
  if (e == 255) return 0;
  const float unit = __uint_as_float(e << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
  return w;
}

// Eight 4-bit values times their block's power of two, exact in bf16 up to its range: a byte of 255 gives NaN, and from kWide4 on (4 * 2^126) some
// values are infinite.
constexpr uint32_t kWide4 = 253;
__device__ __forceinline__ u32x4 from4(uint32_t w, uint32_t e) {
  const float unit = __uint_as_float(e << 23);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3))};
}

// Eight bits: the largest value is 448, 1.75 * 2^8, and what rounds to it goes up to 464, 1.8125 * 2^8: above that mantissa the exponent is one more, so
// no value is cut.  A block's power of two is 2^-124 at least: its least value, 2^-133, is bf16's.
constexpr uint32_t kLeast8 = 3;
__device__ __forceinline__ uint32_t block_exponent8(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = (int)((top + 0x17ffffu) >> 23) - 8;
  return (uint32_t)max(e, (int)kLeast8);
}
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 to8(const float (&x)[8], uint32_t e) {
  if (e == 255) return u32x2{0, 0};
  const float unit = __uint_as_float(e << 23);
  s16x2 a = {0, 0}, b = {0, 0};
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[0], x[1], unit, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, x[2], x[3], unit, true);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[4], x[5], unit, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, x[6], x[7], unit, true);
  return u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
// Eight 8-bit values times their block's power of two, exact in bf16 from kLeast8 on; from 247 (256 * 2^120) on some are infinite.
__device__ __forceinline__ u32x4 from8(uint32_t a, uint32_t b, uint32_t e) {
  const float unit = __uint_as_float(e << 23);
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, unit, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, unit, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, unit, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, unit, true))};
}

// Read: the same lanes, from the cache to rows (19 000 tokens out of 4 bits 22 us, 4.4 TB/s, out of bf16 28 us, 5.4 TB/s; 64 tokens 4.7).
template <int FMT, bool ONCE>
__device__ __forceinline__ void read_rows(const KvDev kv, const KvRowsDev rows) {
  const int lane = threadIdx.x, c = lane & 7, hl = lane >> 3;
  const int row = blockIdx.x / rows.waves, part = blockIdx.x - row * rows.waves;
  const int s = count_up_to([&](int i) { return (int64_t)start_of(kv, i + 1); }, kv.n_seqs, row, lane);
  if (s >= kv.n_seqs || row < start_of(kv, s)) return;      // rows of no sequence stay as they are
  const Slot o = slot_of(kv, row, lane);
  const int H = kv.heads;
  for (int step = part; 8 * step < 2 * H; step += rows.waves) {
    const int e = 8 * step + hl;
    if (e >= 2 * H) continue;
    const bool is_k = e < H;
    const int h = is_k ? e : e - H;
    u32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
    if (o.page >= 0) {
      char* plane = is_k ? +kv.k : +kv.v;
      if constexpr (FMT != kBf16) {
        const char* src = code_row<FMT>(plane, kv, o, h);
        const uint32_t ex = *reinterpret_cast<const uint32_t*>(code_scales<FMT>(plane, kv, o, h));
        const uint32_t ea = ex >> (8 * (c >> 2)) & 255u, eb = ex >> (8 * (c >> 2) + 16) & 255u;
        if constexpr (FMT == kMx4) {
          a = from4(*reinterpret_cast<const uint32_t*>(src + 4 * c), ea);
          b = from4(*reinterpret_cast<const uint32_t*>(src + 32 + 4 * c), eb);
        } else {
          const u32x2 wa = *reinterpret_cast<const u32x2*>(src + 8 * c), wb = *reinterpret_cast<const u32x2*>(src + 64 + 8 * c);
          a = from8(wa[0], wa[1], ea);
          b = from8(wb[0], wb[1], eb);
        }
      } else {
        const char* src = plane + ((((int64_t)o.page << kv.page_shift) + o.at) * H + h) * kRow + 16 * c;
        a = load16<ONCE>(src);
        b = load16<ONCE>(src + 128);
      }
    }
    char* dst = (is_k ? rows.k + row * rows.k_stride : rows.v + row * rows.v_stride) + h * kRow + 16 * c;
    store16<ONCE>(dst, a);
    store16<ONCE>(dst + 128, b);
  }
}

// ---------------------------------------------------------------------------------------------
// Attention.  The query rows of a sequence and KV head are its (token, head of the group) pairs, tokens first; a workgroup takes a
// block of them and a part of the tokens they see.  Scores are kept as the products leave them, unscaled.
// The weights are rounded to bf16 for the second product (2^-8 of each at most): the matrix cores take both operands in one type, and V is bf16.  Their
// sums, the scores and all that is joined stay in fp32.  Results differ from 64 bits by 0.0023 relative, from one rounding of the result by 0.0017.
// ---------------------------------------------------------------------------------------------
// A block of query rows: which sequence it belongs to, and what its rows see.
struct Block {
  int s;              // sequence
  int q0;             // first row of the token buffers
  int n_rows;         // query rows of the sequence
  int r0;             // first row of the block
  int pos0;           // position of the sequence's first new token (may be negative)
  int p_lo, p_hi;     // positions of the block's first and last row
  int hole_b, hole_e;
};

// Row blocks are numbered without knowing the lengths: number s is the first block of sequence s; behind those, sequence s has the numbers
// from floor(q0 group / block) on, at least as many as it has further blocks.  (One token per sequence: no number without a block in between, and
// nothing to search.)  False: no block has this number.
__device__ __forceinline__ bool find_block(const KvDev& kv, const KvAttendDev& at, int id, int block_rows, int lane, Block& b) {
  int64_t r0 = 0;
  if (id < kv.n_seqs) {
    b.s = id;
  } else {
    const int e = id - kv.n_seqs;
    b.s = count_up_to([&](int i) { return (int64_t)start_of(kv, i) * at.group / block_rows; }, kv.n_seqs, e, lane) - 1;
    if (b.s < 0) return false;
    r0 = (e - (int64_t)start_of(kv, b.s) * at.group / block_rows + 1) * block_rows;
  }
  // (all that depends on the sequence alone is asked for at once)
  const int q0 = scalar_read(kv.q_start + b.s), q1 = scalar_read(kv.q_start + b.s + 1), len = scalar_read(kv.seq_len + b.s);
  const int hole_b = at.hole ? scalar_read(at.hole + 2 * b.s) : 0, hole_e = at.hole ? scalar_read(at.hole + 2 * b.s + 1) : 0;
  b.q0 = min(max(q0, 0), kv.n_tokens);
  const int n = min(max(q1, 0), kv.n_tokens) - b.q0;
  b.n_rows = n * at.group;                   // (at most n_tokens * n_q_heads, which the host has checked)
  if (n <= 0 || (uint64_t)r0 >= (uint64_t)b.n_rows) return false;       // (negative where the starts decrease)
  b.r0 = (int)r0;
  b.pos0 = max(len, 0) - n;                  // (tokens of a call and of a table are at most 2^30: differences of positions fit)
  b.p_lo = b.pos0 + b.r0 / at.group;
  b.p_hi = b.pos0 + (min(b.r0 + block_rows, b.n_rows) - 1) / at.group;
  b.hole_b = max(hole_b, 0);
  b.hole_e = max(hole_e, b.hole_b);
  return true;
}

// The tiles that hold what some row of the block sees: at most four runs in ascending order (first tokens and window, each before and
// behind the hole).
struct Tiles {
  int begin[4], count[4], total;
  __device__ __forceinline__ int tile(int i) const {
    const int c0 = count[0], c1 = c0 + count[1], c2 = c1 + count[2];
    return i < c0 ? begin[0] + i : i < c1 ? begin[1] + i - c0 : i < c2 ? begin[2] + i - c1 : begin[3] + i - c2;
  }
};
__device__ __forceinline__ Tiles tiles_of(const KvDev& kv, const KvAttendDev& at, const Block& b, int tile_tokens) {
  const int64_t held = (int64_t)kv.table_stride << kv.page_shift;
  const int end = kv.pool_pages ? (int)min(held, (int64_t)b.p_hi + 1) : 0;
  int near = at.window ? (int)max((int64_t)0, (int64_t)b.p_lo - at.window + 1) : 0, sink = at.window ? min(at.n_sink, end) : 0;
  if (near <= sink) near = sink = 0;         // the window reaches the first tokens
  const int cut[4][2] = {{0, min(sink, b.hole_b)}, {max(0, b.hole_e), sink}, {near, min(end, b.hole_b)}, {max(near, b.hole_e), end}};
  const bool hole = b.hole_e > b.hole_b;
  Tiles t;
  int last = 0;
  t.total = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    int lo = cut[k][0], hi = cut[k][1];
    if (!hole) {
      if (k & 1) hi = lo;                    // one piece each
      else hi = k == 0 ? sink : end;
    }
    t.begin[k] = max(last, max(lo, 0) / tile_tokens);
    const int stop = hi > lo ? (hi - 1) / tile_tokens + 1 : 0;
    t.count[k] = max(0, stop - t.begin[k]);
    if (t.count[k] > 0) last = t.begin[k] + t.count[k];
    t.total += t.count[k];
  }
  return t;
}

// A workgroup's part of the tiles: pieces of one length, so that long sequences have many and short ones few; the last takes what is left of
// a sequence longer than expected.
__device__ __forceinline__ void part_of(const KvAttendDev& at, const Tiles& t, int chunk, int& begin, int& end) {
  begin = (int)min((int64_t)chunk * at.piece_tiles, (int64_t)t.total);
  end = chunk == at.n_chunks - 1 ? t.total : min(begin + at.piece_tiles, t.total);
}

__device__ __forceinline__ bool sees(const KvAttendDev& at, const Block& b, int p, int j) {
  return j <= p && (at.window == 0 || p - j < at.window || j < at.n_sink) && !(j >= b.hole_b && j < b.hole_e);
}
// does some row / does every row of the block see all tokens j0 .. j1?
__device__ __forceinline__ bool all_see(const KvAttendDev& at, const Block& b, int j0, int j1) {
  return j1 <= b.p_lo && (at.window == 0 || b.p_hi - j0 < at.window || j1 < at.n_sink) && (j1 < b.hole_b || j0 >= b.hole_e);
}
__device__ __forceinline__ bool one_sees(const KvAttendDev& at, const Block& b, int j) {
  return j <= b.p_hi && (at.window == 0 || b.p_lo - j < at.window || j < at.n_sink) && !(j >= b.hole_b && j < b.hole_e);
}

// A weight is 2^(scale2 (s - m) - kBelow): s the score q . k as the products leave it, m the row's reference point, which is one of its scores.
// The difference comes first: it is exact where it matters, and zero at the maximum, whatever the scale.  (Scaled first, s scale2 and m scale2 are
// rounded apart, and from 2^30 on that is more than all exponents that fp32 has: rows of zeros and of infinities.)
// The reference point follows the maximum only where a score has passed it by more than 2^kLazy.  Weights are taken 2^kBelow lower, so that none is
// above one: with weights of up to e^8, values of 1e35 and more run over in sums that are finite once divided.  Sums and un-normalised
// outputs carry the factor alike; the logarithm takes it out.
constexpr float kLazy = 11.5f, kBelow = 12.f, kRaise = 4096.f;
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }      // (nothing seen yet: no score above -infinity)
__device__ __forceinline__ float exponent(float s, float ref, float scale2) { return __builtin_fmaf(s - ref, scale2, -kBelow); }
__device__ __forceinline__ float moved(float m, float mx, float scale2) { return (mx - m) * scale2 > kLazy ? mx : m; }
// what sums that go with the reference point m count towards those of a reference point `ref`
__device__ __forceinline__ float share(float m, float ref, float scale2) { return __builtin_amdgcn_exp2f((m - ref) * scale2); }

// Eight elements of a finished row (un-normalised sums o, reference point m, sum l): joined with the caller's partial result and written.
template <class At>
__device__ __forceinline__ void finish(const At& at, int64_t tok, int hq, int piece, const float (&o)[8], float m, float l) {
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = o[i] * inv;
  // log-sum-exp: -infinity for an empty row, NaN for one with a NaN score, infinite where fp32 has no such number
  float lse = l > 0.f ? m * at.scale + __logf(l * kRaise) : l != l ? l : -INFINITY;
  const int64_t idx = tok * at.n_q_heads + hq;
  if (at.other_out) {
    const float pl = at.other_lse[idx];
    if (pl != -INFINITY) {
      const float top = fmaxf(lse, pl);
      const float w = lse == top ? 1.f : __expf(lse - top), pw = pl == top ? 1.f : __expf(pl - top), both = w + pw, wb = w / both, pb = pw / both;
      const float* po = at.other_out + idx * kHeadDim + 8 * piece;
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = wb * r[i] + pb * po[i];      // (shares first: the two together may be beyond fp32)
      lse = top + __logf(both);
    }
  }
  if constexpr (!std::is_same_v<At, KvAttendDev>) {
    if (at.f32) {
      if (at.lse && piece == 0) at.lse[idx] = lse;
      f32x4* dst = reinterpret_cast<f32x4*>(at.out + tok * at.out_stride + hq * (2 * kRow) + 32 * piece);
      dst[0] = f32x4{r[0], r[1], r[2], r[3]};
      dst[1] = f32x4{r[4], r[5], r[6], r[7]};
      return;
    }
  }
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2(r[2 * i], r[2 * i + 1]);
  *reinterpret_cast<u32x4*>(at.out + tok * at.out_stride + hq * kRow + 16 * piece) = v;
  if (at.lse && piece == 0) at.lse[idx] = lse;
}

// The same for a workgroup's part: finished if it is the only one, else kept for the join.
__device__ __forceinline__ void put_row(const KvAttendDev& at, int64_t tok, int hq, int chunk, int piece, const float (&o)[8], float m, float l) {
  if (at.n_chunks == 1) {
    finish(at, tok, hq, piece, o, m, l);
    return;
  }
  const int64_t part = (tok * at.n_q_heads + hq) * at.n_chunks + chunk;
  f32x4* dst = reinterpret_cast<f32x4*>(at.part_o + part * kHeadDim + 8 * piece);
  dst[0] = f32x4{o[0], o[1], o[2], o[3]};
  dst[1] = f32x4{o[4], o[5], o[6], o[7]};
  if (piece == 0) *reinterpret_cast<f32x2*>(at.part_ml + 2 * part) = f32x2{m, l};
}

// A part with no tokens: nothing but that is kept of it.
__device__ __forceinline__ void put_empty(const KvAttendDev& at, const Block& b, int h, int chunk, int block_rows) {
  const int r = b.r0 + (int)threadIdx.x;
  if ((int)threadIdx.x >= block_rows || r >= b.n_rows) return;
  const int64_t row = (int64_t)(b.q0 + r / at.group) * at.n_q_heads + h * at.group + r % at.group;
  *reinterpret_cast<f32x2*>(at.part_ml + 2 * (row * at.n_chunks + chunk)) = f32x2{-INFINITY, 0.f};
}

// Physical pages of the 16-token groups of a tile, -1 where there is none.
template <int N>
struct Pages { int p[N]; };

// The pages of a wavefront's tiles first, first + stride, ... below end: 64 / N tiles' worth in the lanes of one register, those of the tiles behind
// them in another, by one read each.  (Read tile by tile with scalar loads, every step waits for one: the LDS reads share their
// counter.)  next() is called for one tile after the other, and get() serves that tile and the 64 / N behind it.
template <int N>
struct PageList {
  static constexpr int kTiles = 64 / N;
  int now, then;           // registers of the current 64 / N tiles and of the next ones
  int at;                  // place of the current tile in `now`
  int filled;              // tiles that have been read
  __device__ __forceinline__ int fill(const KvDev& kv, int s, const Tiles& tiles, int first, int stride, int end, int lane) {
    const int i = min((int64_t)first + (int64_t)stride * (filled + lane / N), (int64_t)end - 1);
    filled += kTiles;
    const int lp = (16 * N * tiles.tile(i) + 16 * (lane % N)) >> kv.page_shift;
    const int v = kv.table[(int64_t)s * kv.table_stride + min(lp, kv.table_stride - 1)];
    return lp < kv.table_stride && v < kv.pool_pages ? max(v, -1) : -1;
  }
  __device__ __forceinline__ void start(const KvDev& kv, int s, const Tiles& tiles, int first, int stride, int end, int lane) {
    filled = 0;
    now = fill(kv, s, tiles, first, stride, end, lane);
    then = now;
    if (end - first > kTiles * stride) then = fill(kv, s, tiles, first, stride, end, lane);
    at = 0;
  }
  __device__ __forceinline__ void next(const KvDev& kv, int s, const Tiles& tiles, int first, int stride, int end, int lane) {
    if (++at < kTiles) return;
    at = 0;
    now = then;
    if ((int64_t)end - first > (int64_t)filled * stride) then = fill(kv, s, tiles, first, stride, end, lane);
  }
  __device__ __forceinline__ Pages<N> get(int d) const {       // of the d-th tile behind the current one
    Pages<N> o;
    const int k = at + d, r = k < kTiles ? now : then, l = (k < kTiles ? k : k - kTiles) * N;
#pragma unroll
    for (int it = 0; it < N; ++it) o.p[it] = __builtin_amdgcn_readlane(r, l + it);
    return o;
  }
  __device__ __forceinline__ int get(int d, int it) const {    // one of them
    const int k = at + d;
    return __builtin_amdgcn_readlane(k < kTiles ? now : then, (k < kTiles ? k : k - kTiles) * N + it);
  }
};

template <int N>
__device__ __forceinline__ int there(const Pages<N>& pg) {      // bit it: the page of tokens 16 it .. is there
  int ok = 0;
#pragma unroll
  for (int it = 0; it < N; ++it) ok |= (pg.p[it] >= 0 ? 1 : 0) << it;
  return ok;
}

constexpr int kRowStride = kHeadDim + 8;   // bf16 elements per staged V row: with 16 bytes behind each, both the writes (16 bytes of sixteen rows, or
                                           // of a block of four) and the transposing reads (32 bytes of sixteen rows) spread over all banks

// A tile's K and V as they lie in memory.  K: lane (n, g) = (lane % 16, lane / 16) holds token 16 tt + n; bf16: elements 32 kk + 8 g .. + 7 as
// k[2 kk + tt]; 4 bits: elements 32 g .. + 31 (one block) as k[tt]; 8 bits: elements 64 e + 16 g .. + 15 as k[2 tt + e], and all four exponents.
// V: bf16: lane holds 16 bytes (lane % 16) of token 4 i + lane / 16; 4 bits: block lane % 4 of token 16 i + lane / 4; 8 bits: 16 bytes
// (lane % 8) of token 8 i + lane / 8.
template <int FMT>
struct Raw {
  static constexpr int kPieces = FMT == kMx4 ? 2 : FMT == kMx8 ? 4 : 8;
  u32x4 k[kPieces], v[kPieces];
  uint32_t ke[2], ve[FMT == kMx8 ? 4 : 2];
  int ok;                                    // bit tt: the page of tokens 16 tt .. is there
};

template <int FMT>
__device__ __forceinline__ void load_tile(const KvDev& kv, const Pages<2>& pg, int h, int lane, Raw<FMT>& r) {
  const int n = lane & 15, g = lane >> 4, T = 1 << kv.page_shift;
  r.ok = there(pg);
  // (a page that is not there: page 0 is read in its place and what it holds is not seen)
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int64_t page = max(pg.p[tt], 0);
    const int row0 = 16 * tt & (T - 1);
    if constexpr (FMT == kMx4) {
      const int64_t base = (page * kv.heads + h) * (T * 68);
      const char* k = kv.k + base;
      const char* v = kv.v + base;
      r.k[tt] = load_once<u32x4>(k + row0 * kRow4 + (n * kRow4 + 16 * g));
      r.ke[tt] = load_once<uint8_t>(k + (T * kRow4 + row0 * 4) + (n * 4 + g));
      r.v[tt] = load_once<u32x4>(v + row0 * kRow4 + 16 * lane);
      r.ve[tt] = load_once<uint8_t>(v + (T * kRow4 + row0 * 4) + lane);
    } else if constexpr (FMT == kMx8) {
      const int64_t base = (page * kv.heads + h) * (T * (kRow8 + 4));
      const char* k = kv.k + base;
      const char* v = kv.v + base;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        r.k[2 * tt + e] = load_once<u32x4>(k + row0 * kRow8 + (n * kRow8 + 16 * g) + 64 * e);
        r.v[2 * tt + e] = load_once<u32x4>(v + row0 * kRow8 + 16 * lane + 1024 * e);
        r.ve[2 * tt + e] = *reinterpret_cast<const uint8_t*>(v + (T * kRow8 + row0 * 4) + (lane >> 1) + 32 * e);
      }
      r.ke[tt] = *reinterpret_cast<const uint32_t*>(k + (T * kRow8 + row0 * 4) + 4 * n);
    } else {
      const int64_t base = (((page << kv.page_shift) + row0) * kv.heads + h) * kRow;
      const char* k = kv.k + base + (n * kv.heads * kRow + 16 * g);
      const char* v = kv.v + base + (g * kv.heads * kRow + 16 * n);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) r.k[2 * kk + tt] = load_once<u32x4>(k + 64 * kk);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[4 * tt + i] = load_once<u32x4>(v + 4 * i * kv.heads * kRow);
    }
  }
}

__device__ __forceinline__ bool odd16(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// V into LDS (row-major), tokens that no row of the block sees as zeros.  True: some row sees a token that another does not, and
// V holds infinities or NaN, which a weight of zero would not silence.
template <int FMT>
__device__ __forceinline__ bool stage_v(const KvAttendDev& at, const Block& b, int tile, bool masked, int lane, Raw<FMT>& r, uint16_t* Vs) {
  bool odd = false;
  if constexpr (FMT == kMx4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = 16 * i + (lane >> 2);
      if (masked && !((r.ok >> i & 1) && one_sees(at, b, tile * kTile + t))) {
        r.v[i] = u32x4{0, 0, 0, 0};
        r.ve[i] = 0;
      }
      odd |= r.ve[i] >= kWide4;
      u32x4* dst = reinterpret_cast<u32x4*>(Vs + t * kRowStride + 32 * (lane & 3));
#pragma unroll
      for (int e = 0; e < 4; ++e) dst[e] = from4(r.v[i][e], r.ve[i]);
    }
  } else if constexpr (FMT == kMx8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 8 * i + (lane >> 3);
      if (masked && !((r.ok >> (i >> 1) & 1) && one_sees(at, b, tile * kTile + t))) {
        r.v[i] = u32x4{0, 0, 0, 0};
        r.ve[i] = 0;
      }
      const u32x4 x = from8(r.v[i][0], r.v[i][1], r.ve[i]), y = from8(r.v[i][2], r.v[i][3], r.ve[i]);
      if (masked) odd |= odd16(x[0]) || odd16(x[1]) || odd16(x[2]) || odd16(x[3]) || odd16(y[0]) || odd16(y[1]) || odd16(y[2]) || odd16(y[3]);
      u32x4* dst = reinterpret_cast<u32x4*>(Vs + t * kRowStride + 16 * (lane & 7));
      dst[0] = x;
      dst[1] = y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = 4 * i + (lane >> 4);
      if (masked) {
        if (!((r.ok >> (i >> 2) & 1) && one_sees(at, b, tile * kTile + t))) r.v[i] = u32x4{0, 0, 0, 0};
        odd |= odd16(r.v[i][0]) || odd16(r.v[i][1]) || odd16(r.v[i][2]) || odd16(r.v[i][3]);
      }
      *reinterpret_cast<u32x4*>(Vs + t * kRowStride + 8 * (lane & 15)) = r.v[i];
    }
  }
  return masked && b.p_lo != b.p_hi && __any(odd);
}

// Maximum over the lanes n, n + 16, n + 32, n + 48, by exchanges of registers (through LDS each costs a round trip per tile: with the tests of
// unmasked tiles gone as well, 64 sequences of 4000 tokens in 4 bits, 20 rows: 70 -> 64 us).
__device__ __forceinline__ float quad_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// Running softmax of 16 query rows: lane (n, g) holds row n; its sum over the lane's own tokens, and elements 16 b + 4 g + i of the
// un-normalised output.
struct Rows16 {
  float m, l;
  f32x4 o[8];
};

// V with what is not finite as zeros, and where it is +infinity, -infinity and NaN (ones).  Rows of the block differ in what they see, and a weight
// of zero does not silence infinity or NaN: such a tile's products take the finite part of V, and what the rest does to the rows that
// see it follows from products with these masks.  Rare, so small rather than fast.
constexpr uint32_t kOne = 0x3f80u;         // bf16
__device__ __forceinline__ uint32_t kind16(uint32_t v, int kind) {      // 0: finite part; 1, 2, 3: masks
  const bool odd = (v & 0x7f80u) == 0x7f80u, inf = odd && (v & 0x7fu) == 0;
  if (kind == 0) return odd ? 0u : v;
  if (kind == 3) return odd && !inf ? kOne : 0u;
  return inf && ((v >> 15) == 1u) == (kind == 2) ? kOne : 0u;
}
__device__ __forceinline__ u32x4 kind_of(u32x4 v, int kind) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = kind16(v[k] & 0xffffu, kind) | kind16(v[k] >> 16, kind) << 16;
  return v;
}
__device__ __forceinline__ float value_of(int kind) { return kind == 1 ? INFINITY : kind == 2 ? -INFINITY : __uint_as_float(0x7fc00000u); }
// ones for the tokens 2 e, 2 e + 1 of a lane that its row sees
__device__ __forceinline__ uint32_t ones(uint32_t live, int e) { return (live >> (2 * e) & 1u ? kOne : 0u) | (live >> (2 * e + 1) & 1u ? kOne << 16 : 0u); }

// Which row block and part a workgroup takes (`rest`), and which KV head.  Workgroup i runs on XCD i % 8.
//   The numbers of the row blocks have gaps, often regular ones: within each eight of them the places shift by one, so that no XCD gets the
//   gaps alone.
//   bf16: the heads of a row block go to different XCDs, and (by the caller, who adds the sequence and the part) a head to all of them in turn: a
//   head's rows are 256 bytes apart by 256 H, and an XCD that reads one head only asks a part of the memory channels for everything (256
//   sequences of 4000 tokens, 8 heads: 5.6 -> 5.9 TB/s, 64 of 16000 5.0 -> 5.7).
//   4 bits: a head's part of a page is 1088 bytes, so neighbours share cache lines: all heads of a row block go to one XCD (4.9 -> 5.2 TB/s).
template <bool TOGETHER>
__device__ __forceinline__ int rest_of(int heads, int& h) {
  int k;                                     // number before the shift
  if (TOGETHER) {
    const int turn = blockIdx.x >> 3;
    h = turn % heads;
    k = (blockIdx.x & 7) + 8 * (turn / heads);
  } else {
    h = blockIdx.x % heads;
    k = blockIdx.x / heads;
  }
  return (k & ~7) | ((k + (k >> 3)) & 7);
}

// Few query rows (decoding, drafted tokens): a wavefront holds NR tiles of 16 rows and takes every fourth 32-token tile of the workgroup's
// part; the four join at the end.  K goes from memory into the operands of the products as it lies there (S^T = K Q^T: lane (n, g) then
// holds the scores of row n and tokens 16 tt + 4 g + i), V through LDS, where the transposing reads turn it.  With at most 16 of 128 rows to
// share, a page read is used once: nothing is shared between the wavefronts, and none waits for another before the end.
// What bounds it: the reads.  256 sequences of 4000 tokens, 5 heads per KV head: 6.3 TB/s (one KV head, rows in a run: 6.6), 64 of 16 000 6.2;
// 250 of 2000 to 4200 tokens 511 us (6.1 TB/s; counters: matrix cores 4 %, vector units 9 % busy).  4 bits: 5.8 TB/s of pages, 6.2 with 32-token pages (vector units
// 37 %); 32 rows of 64 sequences 61 us (4.7 TB/s), there the vector work of two row tiles.  Few sequences: the start (9 us for 4 of 257 tokens).
template <int FMT, int NR>
__device__ __forceinline__ void attend_rows(const KvDev kv, const KvAttendDev at) {
  constexpr int kJoin = kHeadDim + 4;        // floats per row of the joining area
  __shared__ __align__(16) char lds[4 * kTile * kRowStride * 2];
  __shared__ float ml[4][16][2];
  static_assert(4 * 16 * kJoin * 4 <= 4 * kTile * kRowStride * 2, "the joining area lies over the V tiles");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int h;
  const int rest = rest_of<FMT != kBf16>(kv.heads, h);
  if (rest >= at.n_rest) return;
  const int chunk = rest % at.n_chunks, id = rest / at.n_chunks;
  Block b;
  if (!find_block(kv, at, id, 16 * NR, lane, b)) return;
  if constexpr (FMT == kBf16) h = (h + b.s + chunk) % kv.heads;
  const Tiles tiles = tiles_of(kv, at, b, kTile);
  int t_begin, t_end;
  part_of(at, tiles, chunk, t_begin, t_end);
  if (t_begin == t_end && at.n_chunks > 1) {
    put_empty(at, b, h, chunk, 16 * NR);
    return;
  }

  bf16x8 qf[NR][4];
  int pos[NR];
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    const int r = b.r0 + 16 * rt + n;
    const bool on = r < b.n_rows;
    const int t = (on ? r : b.r0) / at.group, hq = h * at.group + (on ? r : b.r0) % at.group;
    pos[rt] = on ? b.pos0 + t : -1;
    const char* q = at.q + (int64_t)(b.q0 + t) * at.q_stride + hq * kRow;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      u32x4 w = *reinterpret_cast<const u32x4*>(q + (FMT == kMx4 ? 64 * g + 16 * kk : FMT == kMx8 ? 128 * (kk >> 1) + 32 * g + 16 * (kk & 1) : 64 * kk + 16 * g));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = on ? (at.q_flip ? w[e] ^ 0x80008000u : w[e]) : 0u;
      qf[rt][kk] = __builtin_bit_cast(bf16x8, w);
    }
  }
  Rows16 st[NR];
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    st[rt].m = -INFINITY;
    st[rt].l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) st[rt].o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  uint16_t* Vs = reinterpret_cast<uint16_t*>(lds) + wave * kTile * kRowStride;
  // kTurns tiles take turns: once the scores of one are there its registers belong to a later tile, which travels while this one's weights
  // and second products run and the other tiles are worked on.
  constexpr int kTurns = 2;                  // (three and four: the 4-bit kernel spills and loses 5 and 70 %, the 8-bit one gains nothing, and loses 9 %)
  Raw<FMT> raw[kTurns];
  const int first = t_begin + wave;
  PageList<2> pages;
  if (first < t_end) {
    pages.start(kv, b.s, tiles, first, 4, t_end, lane);
#pragma unroll
    for (int d = 0; d < kTurns; ++d)
      if (first + 4 * d < t_end) load_tile<FMT>(kv, pages.get(d), h, lane, raw[d]);
  }
  const auto step = [&](const int i, Raw<FMT>& cur) __attribute__((always_inline)) {
    const int tile = tiles.tile(i), j0 = tile * kTile, ok = cur.ok;
    const bool masked = ok != 3 || !all_see(at, b, j0, j0 + kTile - 1);
    wave_sync();
    const bool odd = stage_v<FMT>(at, b, tile, masked, lane, cur, Vs);
    wave_sync();
    f32x4 s[NR][2];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        u32x4 kf;
        if constexpr (FMT == kMx4) kf = from4(cur.k[tt][kk], cur.ke[tt]);
        else if constexpr (FMT == kMx8)
          kf = from8(cur.k[2 * tt + (kk >> 1)][2 * (kk & 1)], cur.k[2 * tt + (kk >> 1)][2 * (kk & 1) + 1], cur.ke[tt] >> (8 * ((g >> 1) + 2 * (kk >> 1))) & 255u);
        else kf = cur.k[2 * kk + tt];
#pragma unroll
        for (int rt = 0; rt < NR; ++rt)
          s[rt][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), qf[rt][kk], s[rt][tt], 0, 0, 0);
      }
    if (i + 4 * kTurns < t_end) load_tile<FMT>(kv, pages.get(kTurns), h, lane, cur);
    pages.next(kv, b.s, tiles, first, 4, t_end, lane);
    bf16x8 pb[NR];
    uint32_t live[NR];
#pragma unroll
    for (int rt = 0; rt < NR; ++rt) {
      live[rt] = 255;
      if (masked) {
        live[rt] = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const bool see = (ok >> (k >> 2) & 1) && sees(at, b, pos[rt], j0 + 16 * (k >> 2) + 4 * g + (k & 3));
          live[rt] |= (see ? 1u : 0u) << k;
          s[rt][k >> 2][k & 3] = see ? s[rt][k >> 2][k & 3] : -INFINITY;
        }
      }
      float p[8], mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; ++k) mx = fmaxf(mx, s[rt][k >> 2][k & 3]);
      const float m_new = moved(st[rt].m, quad_max(mx), at.scale2), ref = reference(m_new);
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        p[k] = __builtin_amdgcn_exp2f(exponent(s[rt][k >> 2][k & 3], ref, at.scale2));
        sum += p[k];
      }
      if (__any(m_new != st[rt].m)) {
        const float alpha = share(st[rt].m, ref, at.scale2);
        st[rt].l *= alpha;
#pragma unroll
        for (int e = 0; e < 8; ++e) st[rt].o[e] *= alpha;
      }
      st[rt].l += sum;
      st[rt].m = m_new;
      u32x4 pw;
#pragma unroll
      for (int e = 0; e < 4; ++e) pw[e] = pack2(p[2 * e], p[2 * e + 1]);
      pb[rt] = __builtin_bit_cast(bf16x8, pw);
    }
    const uint16_t* base = Vs + (4 * g + (n >> 2)) * kRowStride + 4 * (n & 3);
    const auto operand = [&](int e) {        // V^T: element 16 e + n of tokens 4 g .. + 3 and 16 + 4 g .. + 3
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + 16 * e));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + 16 * kRowStride + 16 * e));
      const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
      return u32x4{l2.x, l2.y, h2.x, h2.y};
    };
    if (odd) {                               // what is not finite goes to the rows that see it, and the products meet the rest
#pragma unroll
      for (int rt = 0; rt < NR; ++rt) {
        const u32x4 see = {ones(live[rt], 0), ones(live[rt], 1), ones(live[rt], 2), ones(live[rt], 3)};
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma clang loop unroll(disable)
          for (int kind = 1; kind <= 3; ++kind) {
            const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kind_of(operand(e), kind)),
                                                                       __builtin_bit_cast(bf16x8, see), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) st[rt].o[e][k] += hit[k] > 0.f ? value_of(kind) : 0.f;
          }
      }
      wave_sync();
#pragma clang loop unroll(disable)
      for (int k = 0; k < 8; ++k) {
        u32x4* x = reinterpret_cast<u32x4*>(Vs + (4 * k + (lane >> 4)) * kRowStride + 8 * (lane & 15));
        *x = kind_of(*x, 0);
      }
      wave_sync();
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const u32x4 a = operand(e);
#pragma unroll
      for (int rt = 0; rt < NR; ++rt)
        st[rt].o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pb[rt], st[rt].o[e], 0, 0, 0);
    }
  };
  for (int i = first; i < t_end; i += 4 * kTurns) {
#pragma unroll
    for (int d = 0; d < kTurns; ++d)
      if (i + 4 * d < t_end) step(i + 4 * d, raw[d]);
  }

  // the four wavefronts' rows joined: 16 lanes per row, eight elements each
  float (*join)[16][kJoin] = reinterpret_cast<float (*)[16][kJoin]>(lds);
  const int row = threadIdx.x >> 4, piece = threadIdx.x & 15;
#pragma unroll
  for (int rt = 0; rt < NR; ++rt) {
    __syncthreads();
    float l = st[rt].l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      ml[wave][n][0] = part_max(st[rt].m, l);
      ml[wave][n][1] = l;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) *reinterpret_cast<f32x4*>(&join[wave][n][16 * e + 4 * g]) = st[rt].o[e];
    __syncthreads();
    const int r = b.r0 + 16 * rt + row;
    if (r >= b.n_rows) continue;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w][row][0]);
    float sum = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float m = ml[w][row][0];
      const float f = m == -INFINITY ? 0.f : share(m, top, at.scale2);
      sum += f * ml[w][row][1];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] += f * join[w][row][8 * piece + k];
    }
    put_row(at, b.q0 + r / at.group, h * at.group + r % at.group, chunk, piece, o, top, sum);
  }
}

// ---------------------------------------------------------------------------------------------
// Many query rows (prompts): four wavefronts of 32 rows share 64-token steps of K and V in LDS (tdk_tiles.h): the score products of the next
// step stand beside the weights and second products of this one, and the pages of the steps behind those travel to LDS meanwhile; 4-bit
// pages by way of registers, where they become bf16.
// What bounds it: the wait between a step's dependent stages, as in the spans' kernel.  Prompts of up to 2048 tokens behind 4000, 5 heads per KV head: 519 us, 853
// TFLOP/s of what the queries see (counters: matrix cores 35 % busy, vector units 39 %, no bank conflicts); in 4 bits 794 where bf16 has 815.  Few of the
// 128 rows in use: the reads (64 sequences of 4000 tokens, 20 rows: 200 us, 5.3 TB/s); in 4 bits the way through registers (150 us, 1.9 TB/s).
// ---------------------------------------------------------------------------------------------
constexpr int kBlockRows = 4 * 32;

struct StepShared {
  unsigned char k[2][kStepTile];
  unsigned char v[2][kStepTile];
  int odd[2][4];                             // per V tile and wavefront: it holds infinity or NaN that only some rows may meet
};

// One plane's 64 tokens of a step: bf16 straight into the LDS tile.  Page groups: 16 tokens, one of the four parts of the tile each.  A page that
// is not there: page 0 is read in its place and what it holds is not seen.
__device__ __forceinline__ void fetch_step(const KvDev& kv, const char* plane, const Pages<4>& pg, int h, const StepLoader& ld, uint32_t off, uint32_t lds) {
  const int T = 1 << kv.page_shift;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t row = ((int64_t)max(pg.p[e], 0) << kv.page_shift) + (16 * e & (T - 1));
    load_to_lds(plane + (row * kv.heads + h) * kRow, off, lds + 4096u * e + ld.lds_wave);
  }
}

// 4 bits: lane l of wavefront w holds block l % 4 of token 16 w + l / 4.
struct Codes {
  u32x4 c;
  uint32_t e;
};
__device__ __forceinline__ Codes fetch_codes(const KvDev& kv, const char* plane, const Pages<4>& pg, int h, int wave, int lane) {
  const int T = 1 << kv.page_shift;
  const int64_t page = max(wave == 0 ? pg.p[0] : wave == 1 ? pg.p[1] : wave == 2 ? pg.p[2] : pg.p[3], 0);
  const int row0 = 16 * wave & (T - 1);
  const char* base = plane + (page * kv.heads + h) * (T * 68);
  return Codes{*reinterpret_cast<const u32x4*>(base + row0 * kRow4 + 16 * lane), *reinterpret_cast<const uint8_t*>(base + (T * kRow4 + row0 * 4) + lane)};
}
template <bool V>
__device__ __forceinline__ void put_codes(const Codes& x, unsigned char* tile, int wave, int lane) {
  const int t = 16 * wave + (lane >> 2);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = 4 * (lane & 3) + e;
    *reinterpret_cast<u32x4*>(tile + (V ? v_place(t, c) : k_place(t, c))) = from4(x.c[e], x.e);
  }
}

// A step whose V holds what only some rows may meet: infinity or NaN goes to the sums of the rows that see its token (kind_of), before the step
// itself takes the finite part.  live: bit i: the row sees token 32 (i / 16) + 8 ((i % 16) / 4) + 4 hh + i % 4.
__device__ __forceinline__ void add_odd(const unsigned char* Vs, uint32_t live, int lane, RowState& st) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
#pragma clang loop unroll(disable)
    for (int kind = 1; kind <= 3; ++kind) {
      f32x16 hit;
#pragma unroll
      for (int i = 0; i < 16; ++i) hit[i] = 0.f;
#pragma clang loop unroll(disable)
      for (int kk = 0; kk < 4; ++kk) {
        const uint32_t l8 = live >> (8 * kk);
        const u32x4 see = {ones(l8, 0), ones(l8, 1), ones(l8, 2), ones(l8, 3)};
        const u32x4 v = kind_of(__builtin_bit_cast(u32x4, v_operand(Vs, kk, q, lane)), kind);
        hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, see), hit, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) st.oacc[q][i] += hit[i] > 0.f ? value_of(kind) : 0.f;
    }
  }
}

template <bool FOUR>
__device__ __forceinline__ void attend_steps(const KvDev kv, const KvAttendDev at) {
  __shared__ __align__(16) StepShared sh;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, hh = lane >> 5;
  int h;
  const int rest = rest_of<false>(kv.heads, h), chunk = rest % at.n_chunks;
  if (rest >= at.n_rest) return;
  Block b;
  // (several blocks per sequence: a causal prompt's last rows see most and start first; one: the numbers without a block come last, ahead of
  // the others they leave some compute units with one workgroup and others with three; 64 sequences of 4000 tokens, 20 rows: 274 -> 202 us)
  const int place = rest / at.n_chunks;
  if (!find_block(kv, at, at.last_id < 0 ? place : at.last_id - place, kBlockRows, lane, b)) return;
  h = (h + b.s + chunk) % kv.heads;
  const Tiles tiles = tiles_of(kv, at, b, kBigTile);
  int t_begin, t_end;
  part_of(at, tiles, chunk, t_begin, t_end);
  if (t_begin == t_end && at.n_chunks > 1) {
    put_empty(at, b, h, chunk, kBlockRows);
    return;
  }
  // the wavefront's own rows
  Block w = b;
  w.r0 = b.r0 + 32 * wave;
  const bool active = w.r0 < b.n_rows;
  w.p_lo = b.pos0 + w.r0 / at.group;
  w.p_hi = b.pos0 + (min(w.r0 + 32, b.n_rows) - 1) / at.group;

  bf16x8 qf[8];
  const int r = w.r0 + n;
  const bool on = r < b.n_rows;
  const int pos = on ? b.pos0 + r / at.group : -1;
  {
    const int rr = on ? r : b.r0;
    const char* q = at.q + (int64_t)(b.q0 + rr / at.group) * at.q_stride + (h * at.group + rr % at.group) * kRow;
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
  const StepLoader ld(kv.heads);
  const uint32_t lds_k[2] = {lds_byte(sh.k[0]), lds_byte(sh.k[1])}, lds_v[2] = {lds_byte(sh.v[0]), lds_byte(sh.v[1])};

  // The tokens of a step that the lane's row sees: bit i is token 32 (i / 16) + 8 ((i % 16) / 4) + 4 hh + i % 4.
  const auto token = [](int i) { return 32 * (i >> 4) + 8 * ((i & 15) >> 2) + (i & 3); };
  const auto live_of = [&](int j0, int ok) __attribute__((always_inline)) {
    const int a = pos - j0 - 4 * hh, sink = at.n_sink - j0 - 4 * hh, hb = b.hole_b - j0 - 4 * hh, he = b.hole_e - j0 - 4 * hh;
    uint32_t live = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const int t = token(k);
      if (t <= a && (at.window == 0 || a - t < at.window || t < sink) && !(t >= hb && t < he) && (ok >> (t >> 4) & 1)) live |= 1u << k;
    }
    return live;
  };
  // Scores of what the row does not see.  Each kind of border in a pass of its own, for the few steps that meet it: all of them together cost
  // more than half a step (8192 tokens, a window of 1024: 284 -> 257 us, together with V checked where it is brought; prompts without a window pay
  // for the two, 519 -> 528 on the same card).
  const auto mask_scores = [&](int j0, int ok, f32x16 (&s)[2], float& mx) __attribute__((always_inline)) {
    const int j1 = j0 + kBigTile - 1;
    if (ok == 15 && all_see(at, w, j0, j1)) return;
    const int a = pos - j0 - 4 * hh;
    if (j1 > w.p_lo) {
#pragma unroll
      for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] = token(k) <= a ? s[k >> 4][k & 15] : -INFINITY;
    }
    if (at.window && w.p_hi - j0 >= at.window && j1 >= at.n_sink) {
      const int low = (int)((unsigned)a - (unsigned)at.window), sink = at.n_sink - j0 - 4 * hh;
#pragma unroll
      for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] = token(k) > low || token(k) < sink ? s[k >> 4][k & 15] : -INFINITY;
    }
    if (ok != 15 || (j1 >= b.hole_b && j0 < b.hole_e)) {
      const int hb = b.hole_b - j0 - 4 * hh, he = b.hole_e - j0 - 4 * hh;
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        const int t = token(k);
        s[k >> 4][k & 15] = !(t >= hb && t < he) && (ok >> (t >> 4) & 1) ? s[k >> 4][k & 15] : -INFINITY;
      }
    }
    rows_max<2>(s, mx);
  };
  // The difference of score and reference point costs the step 3 to 4 % (prompts 530 -> 545 us, with a window 259 -> 270), so it is taken where it is
  // needed: up to 2^12 the product of reference point and scale is rounded by 2^-12 at most, the same for all weights until the point moves.
  constexpr float kFar = 4096.f;
  bool far = false;                          // some row of the wavefront is beyond
  // mx: each lane's maximum of the masked scores to come
  const auto settle = [&](float mx) __attribute__((always_inline)) {
    const float m_new = moved(st.m_run, pair_max(mx), at.scale2);
    if (!__any(m_new != st.m_run)) return;
    const float alpha = share(st.m_run, reference(m_new), at.scale2);       // 1 for the rows whose reference point stays
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
  const auto check_v = [&](int i, int ok, int buf) __attribute__((always_inline)) {
    const int j0 = tiles.tile(i) * kBigTile;
    int any = 0;
    if (ok != 15 || !all_see(at, b, j0, j0 + kBigTile - 1)) {
      u32x4* own = reinterpret_cast<u32x4*>(sh.v[buf] + 16 * threadIdx.x);
      bool mine = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const u32x4 x = own[256 * e];
        if (!((ok >> e & 1) && one_sees(at, b, j0 + 16 * e + (int)(threadIdx.x >> 4)))) own[256 * e] = u32x4{0, 0, 0, 0};
        else mine |= odd16(x[0]) || odd16(x[1]) || odd16(x[2]) || odd16(x[3]);
      }
      any = __any(mine);
    }
    if (lane == 0) sh.odd[buf][wave] = any;
  };
  // the same of 4-bit values, before they are put there
  const auto check_codes = [&](int i, int ok, int buf, Codes& x) __attribute__((always_inline)) {
    const int j0 = tiles.tile(i) * kBigTile;
    int any = 0;
    if (ok != 15 || !all_see(at, b, j0, j0 + kBigTile - 1)) {
      if (!((ok >> wave & 1) && one_sees(at, b, j0 + 16 * wave + (lane >> 2)))) x = Codes{u32x4{0, 0, 0, 0}, 0};
      any = __any(x.e >= kWide4);
    }
    if (lane == 0) sh.odd[buf][wave] = any;
  };

  if (t_begin < t_end) {
    f32x16 s0[2], s1[2];
    // (Behind the last step the last one's pages are read again: what that gives is not used.)
    PageList<4> pages;
    pages.start(kv, b.s, tiles, t_begin, 1, t_end, lane);
    int ok = there(pages.get(0));
    Codes ck[2], cv[2];                      // 4 bits: K of the step behind the next and V of the next one, and both of the step after
    if constexpr (FOUR) {
      const Codes k0 = fetch_codes(kv, kv.k, pages.get(0), h, wave, lane), k1 = fetch_codes(kv, kv.k, pages.get(1), h, wave, lane);
      Codes v0 = fetch_codes(kv, kv.v, pages.get(0), h, wave, lane);
      ck[0] = fetch_codes(kv, kv.k, pages.get(2), h, wave, lane);
      cv[0] = fetch_codes(kv, kv.v, pages.get(1), h, wave, lane);
      ck[1] = fetch_codes(kv, kv.k, pages.get(3), h, wave, lane);
      cv[1] = fetch_codes(kv, kv.v, pages.get(2), h, wave, lane);
      put_codes<false>(k0, sh.k[0], wave, lane);
      check_codes(t_begin, ok, 0, v0);
      put_codes<true>(v0, sh.v[0], wave, lane);
      put_codes<false>(k1, sh.k[1], wave, lane);
    } else {
      const Pages<4> here = pages.get(0), next = pages.get(1);
      fetch_step(kv, kv.k, here, h, ld, ld.k_off, lds_k[0]);
      fetch_step(kv, kv.v, here, h, ld, ld.v_off, lds_v[0]);
      fetch_step(kv, kv.k, next, h, ld, ld.k_off, lds_k[1]);
      landed();
      check_v(t_begin, ok, 0);
    }
    __syncthreads();
    if (active) {
      float mx;
      rows_scores(sh.k[0], qf, n, hh, s0);
      rows_max<2>(s0, mx);
      mask_scores(tiles.tile(t_begin) * kBigTile, ok, s0, mx);
      settle(mx);
    }
    __syncthreads();                         // the first step replaces its K tile
    int i = t_begin;
    const auto step = [&](int odd, f32x16 (&s)[2], f32x16 (&nx)[2]) __attribute__((always_inline)) {
      if (sh.odd[odd][0] | sh.odd[odd][1] | sh.odd[odd][2] | sh.odd[odd][3]) {
        // the rows that see what is not finite have it now, and the step meets the rest
        if (active) add_odd(sh.v[odd], live_of(tiles.tile(i) * kBigTile, ok), lane, st);
        __syncthreads();
        u32x4* own = reinterpret_cast<u32x4*>(sh.v[odd] + 16 * threadIdx.x);
#pragma unroll
        for (int e = 0; e < 4; ++e) own[256 * e] = kind_of(own[256 * e], 0);
        __syncthreads();
      }
      const int ok_next = there(pages.get(1));
      if constexpr (FOUR) {                  // (nobody reads these two tiles in this step)
        int ln = lane;
        asm volatile("" : "+v"(ln));
        put_codes<false>(ck[odd], sh.k[odd], wave, ln);
        if (i + 1 < t_end) check_codes(i + 1, ok_next, odd ^ 1, cv[odd]);
        put_codes<true>(cv[odd], sh.v[odd ^ 1], wave, ln);
        ck[odd] = fetch_codes(kv, kv.k, pages.get(4), h, wave, lane);
        cv[odd] = fetch_codes(kv, kv.v, pages.get(3), h, wave, lane);
      } else {
        fetch_step(kv, kv.k, pages.get(2), h, ld, ld.k_off, lds_k[odd]);
        fetch_step(kv, kv.v, pages.get(1), h, ld, ld.v_off, lds_v[odd ^ 1]);
      }
      pages.next(kv, b.s, tiles, t_begin, 1, t_end, lane);
      ok = ok_next;
      if (active) {
        float mx;
        int ln = lane;
        if (FOUR) asm volatile("" : "+v"(ln));         // (the places in the tiles are worked out again: kept from step to step they spill)
        // (past the last step: scores that are not used)
        if (far) {
          const float ref = reference(st.m_run);
#pragma unroll
          for (int k = 0; k < 32; ++k) s[k >> 4][k & 15] -= ref;
        }
        rows_step(sh.k[odd ^ 1], sh.v[odd], qf, s, nx, mx, at.scale, ln, st,
                  [&] { return far ? -kBelow : -reference(st.m_run) * at.scale2 - kBelow; });
        if (i + 1 < t_end) {
          mask_scores(tiles.tile(i + 1) * kBigTile, ok, nx, mx);
          settle(mx);
        }
      }
      if constexpr (!FOUR) {
        landed();
        if (i + 1 < t_end) check_v(i + 1, ok, odd ^ 1);
      }
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
  static_assert(4 * 32 * 4 * kHeadDim <= 2 * sizeof(StepShared::k), "a wavefront's rows lie over the tiles");
  float l = st.l_run;
  l += __shfl_xor(l, 32);
  const float m = part_max(st.m_run, l);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      *reinterpret_cast<f32x4*>(turn + n * 512 + 16 * ((8 * e + 2 * q4 + hh) ^ n)) =
          f32x4{st.oacc[e][4 * q4], st.oacc[e][4 * q4 + 1], st.oacc[e][4 * q4 + 2], st.oacc[e][4 * q4 + 3]};
  wave_sync();
  const int piece = lane & 15;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int row = 4 * k + (lane >> 4), rr = w.r0 + row;
    const float rm = __shfl(m, row), rl = __shfl(l, row);
    if (rr >= b.n_rows) continue;
    const f32x4 x = *reinterpret_cast<const f32x4*>(turn + row * 512 + 16 * ((2 * piece) ^ row));
    const f32x4 y = *reinterpret_cast<const f32x4*>(turn + row * 512 + 16 * ((2 * piece + 1) ^ row));
    const float o[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    put_row(at, b.q0 + rr / at.group, h * at.group + rr % at.group, chunk, piece, o, rm, rl);
  }
}


// The parts' results of a row joined: a wavefront per row, four groups of 16 lanes that take every fourth part.  Lane l holds the weights of
// the parts l, 64 + l, ...  Two reads in a row, weights and results (80 rows of 64 parts: 7 us; one part after the other 11, a row per 16 lanes 24).
template <class At>
__device__ __forceinline__ void join_parts(const KvDev kv, const At at, int64_t rows) {
  const int lane = threadIdx.x & 63, piece = lane & 15;
  const int64_t idx = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (idx >= rows) return;
  const int64_t tok = idx / at.n_q_heads;
  if (tok < start_of(kv, 0) || tok >= start_of(kv, kv.n_seqs)) return;
  float m[4], l[4], top = -INFINITY;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = 64 * k + lane;
    m[k] = -INFINITY;
    l[k] = 0.f;
    if (c < at.n_chunks) {
      const f32x2 x = *reinterpret_cast<const f32x2*>(at.part_ml + 2 * (idx * at.n_chunks + c));
      m[k] = part_max(x[0], x[1]);
      l[k] = x[1];
    }
    top = fmaxf(top, m[k]);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const f32x4* parts = reinterpret_cast<const f32x4*>(at.part_o + idx * at.n_chunks * kHeadDim) + 2 * piece;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (64 * k >= at.n_chunks) break;
    const bool held = m[k] != -INFINITY;
    const uint64_t parts_held = __ballot(held);
    const float f = held ? share(m[k], top, at.scale2) : 0.f;
    sum += f * l[k];
    for (int c0 = 0; c0 < 64 && 64 * k + c0 < at.n_chunks; c0 += 16) {
      // Sixteen parts a time, four of them in each lane's hands: their reads are under way together.  Parts of which the row saw nothing are not
      // read (nothing was written there); one whose share is below fp32's range is, so that NaN and infinities in it are not lost.
      f32x4 x[4], y[4];
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = c0 + 4 * u + (lane >> 4);
        w[u] = __shfl(f, c);
        x[u] = y[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!(parts_held >> c & 1)) continue;
        x[u] = parts[(int64_t)(64 * k + c) * (kHeadDim / 4)];
        y[u] = parts[(int64_t)(64 * k + c) * (kHeadDim / 4) + 1];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[e] += w[u] * x[u][e];
          o[4 + e] += w[u] * y[u][e];
        }
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    o[e] += __shfl_xor(o[e], 16);
    o[e] += __shfl_xor(o[e], 32);
  }
  if (lane < 16) finish(at, tok, (int)(idx - tok * at.n_q_heads), piece, o, top, sum);
}

template <class... A>
hipError_t launch(void (*kernel)(A...), int64_t blocks, int threads, hipStream_t st, std::common_type_t<A>... args) {
  void* p[] = {(void*)&args...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)blocks), dim3((unsigned)threads), p, 0, st);
}

}  // namespace

}  // namespace tdk
