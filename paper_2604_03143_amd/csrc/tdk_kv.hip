// The kernels of the paged caches in bf16 and in 4 bits (tdk_kv_pages.h has their bodies), and the join of the attention's parts.
#include "tdk_kv_pages.h"

namespace tdk {

// ---------------------------------------------------------------------------------------------
// Append: a token's K and Q heads rotated, its V heads as they are.  Lane (hl, c) = (lane / 8, lane % 8) holds elements 8 c .. + 7 and
// 64 + 8 c .. + 7 of head 8 step + hl of the list K heads, Q heads, V heads: both halves of every pair of either style.
// Every lane evaluates one of the 64 angles in double and passes cosine and sine (rounded to fp32 once) on through LDS: the bits of the rounds'
// tables for any position, with no table to build or read, and no slower for it (12 500 tokens, a wavefront each: 79.3 us, with no angles at all 79.0).
// What bounds it: many tokens, the row writes (12 500 tokens with 40 query heads: 391 MB in 69 us, 5.7 TB/s; the counters show no
// byte more); few, its reads in a row: the starts, the length, the page number (4 tokens 3.7 us, 250 tokens 4.8).
// ---------------------------------------------------------------------------------------------
template <bool FOUR, bool ONCE>
__global__ __launch_bounds__(ONCE && !FOUR ? 256 : 64) void tdk_kv_append_kernel(const KvDev kv, const KvRowsDev rows) {
  __shared__ float2 turn[kHalf];
  // Many tokens, bf16: a workgroup of four wavefronts per token, one of which has the angles (the narrower the window of addresses under way, the
  // faster the writes: 74.5 -> 69.3 us; in 4 bits, with more registers and less to write, 19 000 tokens stored and read back take 116 -> 150,
  // so there one wavefront has a token).  Few tokens: a workgroup per eight heads.
  constexpr bool kWide = ONCE && !FOUR;
  const int lane = threadIdx.x & 63, c = lane & 7, hl = lane >> 3;
  const int row = kWide ? blockIdx.x : blockIdx.x / rows.waves, part = kWide ? threadIdx.x >> 6 : blockIdx.x - row * rows.waves;
  const int parts = kWide ? 4 : rows.waves;
  const int H = kv.heads, HQ = rows.n_q_heads, n = 2 * H + HQ;
  // A step's source rows.  They do not depend on where the token goes: the first step's are asked for before that is looked up, every later
  // one's while the step before it is worked on.
  const auto load = [&](int step, u32x4& a, u32x4& b) __attribute__((always_inline)) {
    const int e = 8 * step + hl;
    a = b = u32x4{0, 0, 0, 0};
    if (e >= n) return;
    const bool is_k = e < H, is_q = !is_k && e < H + HQ;
    const int h = is_k ? e : is_q ? e - H : e - H - HQ;
    const char* src = is_k ? rows.k + row * rows.k_stride : is_q ? rows.q + row * rows.q_stride : rows.v + row * rows.v_stride;
    a = load16<ONCE>(src + h * kRow + 16 * c);
    b = load16<ONCE>(src + h * kRow + 16 * c + 128);
  };
  u32x4 na, nb;
  load(part, na, nb);
  const Slot o = slot_of(kv, row, lane);
  if (o.pos < 0) return;                             // (the queries of a token with no page are rotated all the same)
  if (!kWide || part == 0) {
    double sn, cs;
    sincos((double)o.pos * rows.inv_freq[lane], &sn, &cs);
    turn[lane] = make_float2((float)cs, (float)sn);
  }
  if (kWide) __syncthreads();
  else wave_sync();
  float2 t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = turn[kv.interleaved ? 4 * c + (i & 3) + 32 * (i >> 2) : 8 * c + i];
  for (int step = part; 8 * step < n; step += parts) {
    const int e = 8 * step + hl;
    const bool is_k = e < H, is_q = !is_k && e < H + HQ, on = e < n;
    const int h = is_k ? e : is_q ? e - H : e - H - HQ;
    u32x4 a = na, b = nb;
    load(step + parts, na, nb);
    if (!FOUR && !is_k && !is_q) {                   // values move as they are
      if (!on || o.page < 0) continue;
      char* dst = kv.v + ((((int64_t)o.page << kv.page_shift) + o.at) * H + h) * kRow + 16 * c;
      store16<ONCE>(dst, a);
      store16<ONCE>(dst + 128, b);
      continue;
    }
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = lo16(a[i]); x[2 * i + 1] = hi16(a[i]);
      y[2 * i] = lo16(b[i]); y[2 * i + 1] = hi16(b[i]);
    }
    if (is_k || is_q) {
      if (kv.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float xa = x[2 * i], xb = x[2 * i + 1], ya = y[2 * i], yb = y[2 * i + 1];
          x[2 * i] = __builtin_fmaf(xa, t[i].x, -(xb * t[i].y));
          x[2 * i + 1] = __builtin_fmaf(xb, t[i].x, xa * t[i].y);
          y[2 * i] = __builtin_fmaf(ya, t[4 + i].x, -(yb * t[4 + i].y));
          y[2 * i + 1] = __builtin_fmaf(yb, t[4 + i].x, ya * t[4 + i].y);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float xa = x[i], xb = y[i];
          x[i] = __builtin_fmaf(xa, t[i].x, -(xb * t[i].y));
          y[i] = __builtin_fmaf(xb, t[i].x, xa * t[i].y);
        }
      }
    }
    if (!FOUR || is_q) {
      if (!on || (is_k && o.page < 0)) continue;
      char* dst = is_q ? rows.q_out + row * rows.q_out_stride + h * kRow : kv.k + ((((int64_t)o.page << kv.page_shift) + o.at) * H + h) * kRow;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = pack2(x[2 * i], x[2 * i + 1]);
        b[i] = pack2(y[2 * i], y[2 * i + 1]);
      }
      store16<ONCE>(dst + 16 * c, a);
      store16<ONCE>(dst + 16 * c + 128, b);
    } else {
      // (lanes of one block always take the same way here: they hold the same head)
      const uint32_t ex = block_exponent(top_bits(x)), ey = block_exponent(top_bits(y));
      const uint32_t wx = to4(x, ex), wy = to4(y, ey);
      const uint32_t ex1 = (uint32_t)__shfl_xor((int)ex, 4), ey1 = (uint32_t)__shfl_xor((int)ey, 4);
      if (!on || o.page < 0) continue;
      char* dst = code_row<kMx4>(is_k ? kv.k : kv.v, kv, o, h);
      *reinterpret_cast<uint32_t*>(dst + 4 * c) = wx;
      *reinterpret_cast<uint32_t*>(dst + 32 + 4 * c) = wy;
      if (c == 0) *reinterpret_cast<uint32_t*>(code_scales<kMx4>(is_k ? kv.k : kv.v, kv, o, h)) = ex | ex1 << 8 | ey << 16 | ey1 << 24;
    }
  }
}

template <bool FOUR, bool ONCE>
__global__ __launch_bounds__(64) void tdk_kv_read_kernel(const KvDev kv, const KvRowsDev rows) {
  read_rows<FOUR ? kMx4 : kBf16, ONCE>(kv, rows);
}

template <bool FOUR, int NR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(FOUR && NR == 1 ? 3 : 2, FOUR && NR == 1 ? 3 : 2))) void tdk_kv_attend_rows_kernel(const KvDev kv, const KvAttendDev at) {
  attend_rows<FOUR ? kMx4 : kBf16, NR>(kv, at);
}

template <bool FOUR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void tdk_kv_attend_tile_kernel(const KvDev kv, const KvAttendDev at) {
  attend_steps<FOUR>(kv, at);
}

__global__ __launch_bounds__(256) void tdk_kv_attend_join_kernel(const KvDev kv, const KvAttendDev at, int64_t rows) { join_parts(kv, at, rows); }

// (many tokens pass the caches by: 12 500 tokens 79 -> 74 us, 19 000 in 4 bits and back 132 -> 118.  Few stay there, also where a wavefront has all of a
// token: 250 tokens of four heads without queries, attention to 300 tokens each behind it, 38.5 -> 38.2 us together; of 1500
// tokens the append 5.0 -> 4.2, with attention 180 -> 185)
hipError_t launch_kv_append(const KvDev& kv, const KvRowsDev& rows, int fmt, bool many, hipStream_t st) {
  if (fmt == kMx8 || rows.rotary != kHeadDim || rows.magnitude != 1.0) return launch_kv_append_rope(kv, rows, fmt, many, st);
  const bool four = fmt == kMx4;
  auto kernel = many ? (four ? tdk_kv_append_kernel<true, true> : tdk_kv_append_kernel<false, true>)
                     : (four ? tdk_kv_append_kernel<true, false> : tdk_kv_append_kernel<false, false>);
  return launch(kernel, (int64_t)kv.n_tokens * rows.waves, many && !four ? 256 : 64, st, kv, rows);
}

hipError_t launch_kv_read(const KvDev& kv, const KvRowsDev& rows, int fmt, bool many, hipStream_t st) {
  if (fmt == kMx8) return launch_kv8_read(kv, rows, many, st);
  const bool four = fmt == kMx4;
  auto kernel = many ? (four ? tdk_kv_read_kernel<true, true> : tdk_kv_read_kernel<false, true>)
                     : (four ? tdk_kv_read_kernel<true, false> : tdk_kv_read_kernel<false, false>);
  return launch(kernel, (int64_t)kv.n_tokens * rows.waves, 64, st, kv, rows);
}

hipError_t launch_kv_join(const KvDev& kv, const KvAttendDev& at, int64_t rows, hipStream_t st) {
  return launch(tdk_kv_attend_join_kernel, (rows + 3) / 4, 256, st, kv, at, rows);
}

hipError_t launch_kv_attend(const KvDev& kv, const KvAttendDev& at, const KvAttendPlan& p, int fmt, hipStream_t st) {
  const int64_t blocks = (p.ids * p.n_chunks + 7) / 8 * 8 * kv.heads;
  const bool four = fmt == kMx4;
  hipError_t e;
  if (fmt == kMx8) {
    e = launch_kv8_attend(kv, at, p, blocks, st);
  } else if (p.block_rows == 128) {
    e = launch(four ? tdk_kv_attend_tile_kernel<true> : tdk_kv_attend_tile_kernel<false>, blocks, 256, st, kv, at);
  } else {
    auto kernel = p.block_rows == 32 ? tdk_kv_attend_rows_kernel<true, 2> : four ? tdk_kv_attend_rows_kernel<true, 1> : tdk_kv_attend_rows_kernel<false, 1>;
    e = launch(kernel, blocks, 256, st, kv, at);
  }
  return e == hipSuccess && p.n_chunks > 1 ? launch_kv_join(kv, at, p.rows, st) : e;
}

}  // namespace tdk
