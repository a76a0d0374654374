// The kernels of the paged caches in 8 bits (tdk_rope.hip has the append).
#include "tdk_steps.h"

namespace tdk {

namespace {

// Pages in 8 bits by way of registers, where they become bf16.  Lane l of wavefront w brings 16 bytes (l % 8) of the tokens 16 w + 8 i + l / 8 of
// a step: what is written to LDS at a step's start was asked for at the start of the one before.
struct Codes8 {
  u32x4 c[2];
  uint32_t e[2];                             // their exponents
};

constexpr uint32_t kWide8 = 247;             // from this power on a block's values may be infinite

struct PageSource {
  using At = KvAttendDev;
  static constexpr bool kHoles = true, kSpread = false, kEnds = false;      // (a test whether there is a next step: 40 rows 132 -> 148 us)
  static __device__ __forceinline__ bool wide(const At&) { return false; }

  Tiles tiles;
  int total;
  __device__ __forceinline__ bool find(const KvDev& kv, const At& at, int place, int lane, Block& b) {
    if (!find_block(kv, at, at.last_id < 0 ? place : at.last_id - place, kRows, lane, b)) return false;
    tiles = tiles_of(kv, at, b, kStep);
    total = tiles.total;
    return true;
  }

  const KvDev* cache;
  const At* a;
  const Block* blk;
  StepTiles* sh;
  PageList<4> pages;
  Codes8 ck, cv;
  int t_begin, t_end, wave, lane;
  const char *codes_k, *codes_v;             // of page 0: the wavefront's tokens
  uint32_t page_bytes, powers;               // powers: where they stand behind the codes
  uint32_t put_k, put_v;                     // the first of the lane's places in a tile
  // of the d-th step behind the current one
  __device__ __forceinline__ Codes8 fetch(const char* plane, int d) const {
    const char* c = plane + (uint64_t)(uint32_t)max(pages.get(d, wave), 0) * page_bytes;
    const char* e = c + powers;
    const uint32_t off = 16u * (uint32_t)lane, off_e = (uint32_t)lane >> 1;
    Codes8 x;
    x.c[0] = *reinterpret_cast<const u32x4*>(c + off);
    x.c[1] = *reinterpret_cast<const u32x4*>(c + off + 1024);
    x.e[0] = *reinterpret_cast<const uint8_t*>(e + off_e);
    x.e[1] = *reinterpret_cast<const uint8_t*>(e + off_e + 32);
    return x;
  }
  template <bool V>
  __device__ __forceinline__ void put(const Codes8& x, unsigned char* tile) const {
    uint32_t at = V ? put_v : put_k;
    asm volatile("" : "+v"(at));             // (the other places are worked out from the first: kept from step to step they spill)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e)            // (token + 8: K's rows place their pieces by four bits of it, V's by two)
        *reinterpret_cast<u32x4*>(tile + ((at ^ (16 * e) ^ (V ? 0 : 128 * i)) + 2048 * i)) = from8(x.c[i][2 * e], x.c[i][2 * e + 1], x.e[i]);
  }
  // V of a step that some rows see and some do not, before it is put there: what none sees becomes zero (a weight of zero would not silence infinity
  // or NaN), and the tile's flag says whether what is left is finite.
  __device__ __forceinline__ void check(int i, int there, int place, Codes8& x) const {
    const int j0 = tiles.tile(i) * kStep, near = a->window ? a->window : INT32_MAX;
    uint32_t nan = 0, power = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = j0 + 16 * wave + 8 * k + (lane >> 3);
      const bool seen = (there >> wave & 1) & (j <= blk->p_hi) & ((blk->p_lo - j < near) | (j < a->n_sink)) & !((j >= blk->hole_b) & (j < blk->hole_e));
      x.e[k] = seen ? x.e[k] : 0;
      power = max(power, x.e[k]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x.c[k][e] = seen ? x.c[k][e] : 0;
        nan |= (x.c[k][e] & 0x7f7f7f7fu) + 0x01010101u;       // bit 7 of a byte: its code is NaN
      }
    }
    const int any = __any((nan & 0x80808080u) != 0 || power >= kWide8);
    if (lane == 0) sh->odd[place][wave] = any;
  }
  __device__ __forceinline__ void open(const KvDev& kv, const At& at, const Block& b, int head, int begin, int end, StepTiles& to, int lane_, int wave_) {
    cache = &kv;
    a = &at;
    blk = &b;
    sh = &to;
    t_begin = begin;
    t_end = end;
    lane = lane_;
    wave = wave_;
    const int T = 1 << kv.page_shift, row0 = 16 * wave & (T - 1);
    page_bytes = (uint32_t)(kv.heads * T * (kRow8 + 4));
    powers = (uint32_t)(T * kRow8 + row0 * 4 - row0 * kRow8);
    codes_k = kv.k + (int64_t)head * (T * (kRow8 + 4)) + row0 * kRow8;
    codes_v = kv.v + (int64_t)head * (T * (kRow8 + 4)) + row0 * kRow8;
    put_k = (uint32_t)k_place(16 * wave + (lane >> 3), 2 * (lane & 7));
    put_v = (uint32_t)v_place(16 * wave + (lane >> 3), 2 * (lane & 7));
    // (Behind the last step the last one's pages are read again: what that gives is not used.)
    if (begin < end) pages.start(kv, b.s, tiles, begin, 1, end, lane);
  }
  __device__ __forceinline__ int token(int i) const { return tiles.tile(i) * kStep; }
  __device__ __forceinline__ int ok(int d) const { return there(pages.get(d)); }      // of the d-th step behind the current one
  __device__ __forceinline__ bool seen(int i, int there) const {
    const int j0 = token(i);
    return there == 15 && all_see(*a, *blk, j0, j0 + kStep - 1);
  }
  __device__ __forceinline__ bool whole(int i, int d) const { return seen(i, ok(d)); }
  __device__ __forceinline__ void first() {
    const Codes8 k0 = fetch(codes_k, 0), k1 = fetch(codes_k, 1);
    Codes8 v0 = fetch(codes_v, 0);
    ck = fetch(codes_k, 2);
    cv = fetch(codes_v, 1);
    put<false>(k0, sh->k[1]);
    const int there0 = ok(0);
    if (!seen(t_begin, there0)) check(t_begin, there0, 0, v0);
    put<true>(v0, sh->v[0]);
    put<false>(k1, sh->k[0]);
  }
  __device__ __forceinline__ void bring(int i, int place, bool to_check) {
    put<false>(ck, sh->k[place]);
    if (to_check) check(i + 1, ok(1), place, cv);
    put<true>(cv, sh->v[place]);
    ck = fetch(codes_k, 3);
    cv = fetch(codes_v, 2);
    pages.next(*cache, blk->s, tiles, t_begin, 1, t_end, lane);
  }
  __device__ __forceinline__ void arrived(int, int, bool) const {}
};

}  // namespace

// Read: 20 851 tokens (8 heads) 27 us, 4.8 TB/s of codes read and bf16 written; 250 tokens 2.9.  What bounds it is the order of a wavefront's reads, not yet memory (a copy has
// 6.7): the sequence is searched twice, one search behind the other (read_rows, slot_of), and a step's codes are asked for when those before are written.
template <bool ONCE>
__global__ __launch_bounds__(64) void tdk_kv8_read_kernel(const KvDev kv, const KvRowsDev rows) {
  read_rows<kMx8, ONCE>(kv, rows);
}

// Up to 32 rows of a sequence and KV head: the rows kernel of the other formats (attend_rows).  A lane's 16 bytes of K are half a block: they become bf16 right before
// their products, with the block's power of two in the same conversions, and the inner dimension runs in that order.
// What bounds it: the codes' way from memory.  250 tokens over 2000 to 4200 each: 280 us, 5.65 TB/s (32-token pages 5.9), fetched 2 % more than they hold; 20 rows over 64 sequences of
// 4000 tokens 89 us.  The exponents' cache lines serve neighbouring tokens' lanes again, so they stay in the caches: 287 -> 280 us (past them, as the codes).  Tried:
// three wavefronts per SIMD spill (450 us), three register sets gain nothing and four lose 9 %, codes through the caches lose 2 to 6 %.
template <int NR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_kv8_attend_rows_kernel(const KvDev kv, const KvAttendDev at) {
  attend_rows<kMx8, NR>(kv, at);
}

// More rows: attend_in_steps.  Prompts of up to 2048 tokens behind 4000, 5 queries a head: 469 to 496 us by card, 842 to 890 TFLOP/s; four whole ones 949 (a prompt whose
// rows need no conversion: 1043 to 1121).  Bounded by vector instructions, a fifth of which bring the pages (46 % busy, matrix cores 39 %), and by unequal blocks in three rounds of
// workgroups.  Fewer instructions there made it faster: a wavefront asks for its own page alone (507 -> 493 us), works out a lane's four places in a tile from
// one (-> 484), sees by codes and powers whether V is finite (492 -> 481 on another card); an order of the writes without bank conflicts (10 % of LDS's time) costs more than it saves.  The body without the pipeline that paged
// bf16 has took 669 us for 515 at the time.  40 rows over 64 sequences of 4000 tokens: 118 us.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_kv8_attend_tile_kernel(const KvDev kv, const KvAttendDev at) {
  attend_in_steps<PageSource>(kv, at);
}

hipError_t launch_kv8_read(const KvDev& kv, const KvRowsDev& rows, bool many, hipStream_t st) {
  return launch(many ? tdk_kv8_read_kernel<true> : tdk_kv8_read_kernel<false>, (int64_t)kv.n_tokens * rows.waves, 64, st, kv, rows);
}

hipError_t launch_kv8_attend(const KvDev& kv, const KvAttendDev& at, const KvAttendPlan& p, int64_t blocks, hipStream_t st) {
  if (p.block_rows == 128) return launch(tdk_kv8_attend_tile_kernel, blocks, 256, st, kv, at);
  return launch(p.block_rows == 32 ? tdk_kv8_attend_rows_kernel<2> : tdk_kv8_attend_rows_kernel<1>, blocks, 256, st, kv, at);
}

}  // namespace tdk
