// Rotation by the frequencies of a handle: rows that stay rows, and rows on their way into a cache where part of the head turns, cosines
// and sines have a magnitude, or the pages have 8 bits.
#include "tdk_kv_pages.h"

namespace tdk {

namespace {

// cosine and sine of the lane's angle (lane j: pair j), rounded to fp32 once
__device__ __forceinline__ float2 angle_of(int pos, double freq, double cos_size, double sin_size) {
  double sn, cs;
  sincos((double)pos * freq, &sn, &cs);
  return make_float2((float)(cs * cos_size), (float)(sn * sin_size));
}

__device__ __forceinline__ void turn_pair(float& a, float& b, float2 t) {
  const float xa = a, xb = b;
  a = __builtin_fmaf(xa, t.x, -(xb * t.y));
  b = __builtin_fmaf(xb, t.x, xa * t.y);
}

__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = lo16(w[i]);
    x[2 * i + 1] = hi16(w[i]);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// Rotate: K and Q heads of a token, eight heads per wavefront and step, eight lanes per head.  A lane holds two pieces of 16 bytes, chosen so that a pair
// never crosses lanes.  R elements turn, in pieces of eight: half layout: the lanes c < R / 16 hold the pieces c and c + R / 16, the others two of
// the pieces behind, which pass as they are; interleaved: pieces c and c + 8, of which those below R / 8 turn.
// Angles as in the append: one per lane, in double, rounded to fp32 once; a pair turns in fp32 and is rounded to bf16 once.
// What bounds it: memory.  12 333 tokens (8 + 40 heads): 51 us, 5.9 TB/s; 32 768: 129 us, 6.2 TB/s; 40 000 with 24 heads, half of each: 75 us, 5.9 TB/s; reads and writes pass the caches by.  Four tokens: 3.7 us, of which the launch
// is most.  Up to four wavefronts, one for each eight heads, share a token's angles where there are many tokens (many_rows; always four: 16 heads 66 us for 51); few
// tokens have a workgroup for each eight heads.
// ---------------------------------------------------------------------------------------------
template <bool MANY, bool ONCE>
__global__ __launch_bounds__(MANY ? 256 : 64) void tdk_kv_rotate_kernel(const KvDev kv, const KvRotateDev r) {
  __shared__ float2 turn[kHalf];
  const int lane = threadIdx.x & 63, c = lane & 7, hl = lane >> 3;
  const int row = MANY ? blockIdx.x : blockIdx.x / r.waves, part = MANY ? threadIdx.x >> 6 : blockIdx.x - row * r.waves;
  const int parts = r.waves;
  const int H = r.n_k_heads, n = H + r.n_q_heads;
  const int R16 = r.rotary >> 4;
  const int pa = kv.interleaved ? c : c < R16 ? c : R16 + c, pb = kv.interleaved ? c + 8 : c < R16 ? c + R16 : 8 + c;
  const bool turn_a = kv.interleaved ? pa < 2 * R16 : c < R16, turn_b = kv.interleaved ? pb < 2 * R16 : c < R16;
  const char* const k = r.k + row * r.k_stride;
  const char* const q = r.q + row * r.q_stride;
  const auto load = [&](int step, u32x4& a, u32x4& b) __attribute__((always_inline)) {
    const int e = 8 * step + hl;
    a = b = u32x4{0, 0, 0, 0};
    if (e >= n) return;
    const char* src = e < H ? k + e * kRow : q + (e - H) * kRow;
    a = load16<ONCE>(src + 16 * pa);
    b = load16<ONCE>(src + 16 * pb);
  };
  u32x4 na, nb;
  load(part, na, nb);
  const Slot o = slot_of(kv, row, lane);
  if (o.pos < 0) return;
  if (!MANY || part == 0) turn[lane] = angle_of(o.pos, r.inv_freq[lane], r.cos_size, r.sin_size);
  if (MANY) __syncthreads();
  else wave_sync();
  float2 t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = turn[kv.interleaved ? 4 * c + (i & 3) + 32 * (i >> 2) : 8 * c + i];
  char* const k_out = r.k_out + row * r.k_out_stride;
  char* const q_out = r.q_out + row * r.q_out_stride;
  for (int step = part; 8 * step < n; step += parts) {
    const int e = 8 * step + hl;
    u32x4 a = na, b = nb;
    load(step + parts, na, nb);
    if (e >= n) continue;
    float x[8], y[8];
    unpack8(a, x);
    unpack8(b, y);
    if (kv.interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        turn_pair(x[2 * i], x[2 * i + 1], t[i]);
        turn_pair(y[2 * i], y[2 * i + 1], t[4 + i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn_pair(x[i], y[i], t[i]);
    }
    char* dst = e < H ? k_out + e * kRow : q_out + (e - H) * kRow;
    store16<ONCE>(dst + 16 * pa, turn_a ? pack8(x) : a);
    store16<ONCE>(dst + 16 * pb, turn_b ? pack8(y) : b);
  }
}

// ---------------------------------------------------------------------------------------------
// Append, the forms that tdk_kv_append_kernel does not have: lanes and steps as there.  A piece whose pair lies in another lane (half layout, part of the
// head) gets its partner by exchanges: piece k < R / 8 pairs with the one R / 16 further on, or back.
// What bounds it: writes that lie scattered.  20 851 tokens into 8-bit pages (8 + 64 heads): 143 us, 5.7 TB/s; 250 tokens 5.1 us.  One wavefront per token: with four,
// as the rotation has them, the call took 183 us instead of 172 together with the read behind it.  Half of the head, or a magnitude, 20 000 tokens of 8 + 40 heads: into bf16
// pages 103 us, 5.55 TB/s (plain rotation, four wavefronts per token: 100 us, 5.7), into 4 bits 92 to 95, 5.4 to 5.6 (plain 97); 12 500 tokens 68 (65) and 62 to 64 (65).
// ---------------------------------------------------------------------------------------------
template <int FMT, bool ONCE>
__global__ __launch_bounds__(64) void tdk_kv_append_rope_kernel(const KvDev kv, const KvRowsDev rows) {
  __shared__ float2 turn[kHalf];
  const int lane = threadIdx.x, c = lane & 7, hl = lane >> 3;
  const int row = blockIdx.x / rows.waves, part = blockIdx.x - row * rows.waves;
  const int H = kv.heads, HQ = rows.n_q_heads, n = 2 * H + HQ, R16 = rows.rotary >> 4;
  const char* const src_k = rows.k + row * rows.k_stride + 16 * c;
  const char* const src_v = rows.v + row * rows.v_stride + 16 * c;
  const char* const src_q = rows.q + row * rows.q_stride + 16 * c;
  const auto load = [&](int step, u32x4& a, u32x4& b) __attribute__((always_inline)) {
    const int e = 8 * step + hl;
    a = b = u32x4{0, 0, 0, 0};
    if (e >= n) return;
    const char* src = e < H ? src_k + e * kRow : e < H + HQ ? src_q + (e - H) * kRow : src_v + (e - H - HQ) * kRow;
    a = load16<ONCE>(src);
    b = load16<ONCE>(src + 128);
  };
  u32x4 na, nb;
  load(part, na, nb);
  const Slot o = slot_of(kv, row, lane);
  if (o.pos < 0) return;                             // (the queries of a token with no page are rotated all the same)
  turn[lane] = angle_of(o.pos, rows.inv_freq[lane], rows.magnitude, rows.magnitude);
  wave_sync();
  const bool part_half = !kv.interleaved && R16 < 8;
  // places of the pieces c and c + 8, and of their partners
  const auto partner = [&](int k) { return k < R16 ? k + R16 : k < 2 * R16 ? k - R16 : k; };
  const int fa = partner(c), fb = partner(c + 8);
  float2 t[8], u[8];                                 // (u: part of the head, half layout: of the piece c + 8)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    t[i] = turn[kv.interleaved ? 4 * c + (i & 3) + 32 * (i >> 2) : part_half ? (8 * min(c, fa) + i) & 63 : 8 * c + i];
    u[i] = turn[(8 * min(c + 8, fb) + i) & 63];
  }
  char* const q_out = rows.q_out + row * rows.q_out_stride;
  for (int step = part; 8 * step < n; step += rows.waves) {
    const int e = 8 * step + hl;
    const bool is_k = e < H, is_q = !is_k && e < H + HQ, on = e < n;
    const int h = is_k ? e : is_q ? e - H : e - H - HQ;
    u32x4 a = na, b = nb;
    load(step + rows.waves, na, nb);
    float x[8], y[8];
    unpack8(a, x);
    unpack8(b, y);
    bool same_a = true, same_b = true;               // these pieces move as they are
    if (is_k || is_q) {
      same_a = c >= 2 * R16;
      same_b = c + 8 >= 2 * R16;
      if (kv.interleaved) {
        if (!same_a) {
#pragma unroll
          for (int i = 0; i < 4; ++i) turn_pair(x[2 * i], x[2 * i + 1], t[i]);
        }
        if (!same_b) {
#pragma unroll
          for (int i = 0; i < 4; ++i) turn_pair(y[2 * i], y[2 * i + 1], t[4 + i]);
        }
      } else if (!part_half) {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn_pair(x[i], y[i], t[i]);
      } else {
        // (a head's eight lanes take the same way here)
        u32x4 pa, pb;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t va = __shfl(a[i], (lane & ~7) | (fa & 7)), vb = __shfl(b[i], (lane & ~7) | (fa & 7));
          pa[i] = fa < 8 ? va : vb;
          const uint32_t wa = __shfl(a[i], (lane & ~7) | (fb & 7)), wb = __shfl(b[i], (lane & ~7) | (fb & 7));
          pb[i] = fb < 8 ? wa : wb;
        }
        float p[8], q[8];
        unpack8(pa, p);
        unpack8(pb, q);
        if (!same_a) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(x[i], t[i].x, c < R16 ? -(p[i] * t[i].y) : p[i] * t[i].y);
        }
        if (!same_b) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(y[i], u[i].x, q[i] * u[i].y);      // (a second member always: R16 < 8)
        }
      }
    }
    if (FMT == kBf16 || is_q) {
      if (!on || (!is_q && o.page < 0)) continue;
      char* dst = is_q ? q_out + h * kRow : (is_k ? +kv.k : +kv.v) + ((((int64_t)o.page << kv.page_shift) + o.at) * H + h) * kRow;
      store16<ONCE>(dst + 16 * c, same_a ? a : pack8(x));
      store16<ONCE>(dst + 16 * c + 128, same_b ? b : pack8(y));
    } else {
      // (lanes of one block always take the same way here: they hold the same head)
      const uint32_t tx = top_bits(x), ty = top_bits(y);
      const uint32_t ex = FMT == kMx4 ? block_exponent(tx) : block_exponent8(tx), ey = FMT == kMx4 ? block_exponent(ty) : block_exponent8(ty);
      const uint32_t ex1 = (uint32_t)__shfl_xor((int)ex, 4), ey1 = (uint32_t)__shfl_xor((int)ey, 4);
      if (!on || o.page < 0) continue;
      char* const plane = is_k ? +kv.k : +kv.v;
      char* dst = code_row<FMT>(plane, kv, o, h);
      if constexpr (FMT == kMx4) {
        *reinterpret_cast<uint32_t*>(dst + 4 * c) = to4(x, ex);
        *reinterpret_cast<uint32_t*>(dst + 32 + 4 * c) = to4(y, ey);
      } else if constexpr (FMT == kMx8) {
        *reinterpret_cast<u32x2*>(dst + 8 * c) = to8(x, ex);
        *reinterpret_cast<u32x2*>(dst + 64 + 8 * c) = to8(y, ey);
      }
      if (c == 0) *reinterpret_cast<uint32_t*>(code_scales<FMT>(plane, kv, o, h)) = ex | ex1 << 8 | ey << 16 | ey1 << 24;
    }
  }
}

// (Half layout, part of the head: the pieces are not whole cache lines, which past the caches would travel twice: 40 000 tokens, 24 heads, 64 of 128: 92 us,
// through the caches 84; 16 of 128: 98 and 83.)
hipError_t launch_kv_rotate(const KvDev& kv, const KvRotateDev& r, bool many, hipStream_t st) {
  if (!many) return launch(tdk_kv_rotate_kernel<false, false>, (int64_t)kv.n_tokens * r.waves, 64, st, kv, r);
  return launch(kv.interleaved || r.rotary == kHeadDim ? tdk_kv_rotate_kernel<true, true> : tdk_kv_rotate_kernel<true, false>, kv.n_tokens, 64 * r.waves, st, kv, r);
}

hipError_t launch_kv_append_rope(const KvDev& kv, const KvRowsDev& rows, int fmt, bool many, hipStream_t st) {
  auto kernel = fmt == kMx8   ? (many ? tdk_kv_append_rope_kernel<kMx8, true> : tdk_kv_append_rope_kernel<kMx8, false>)
                : fmt == kMx4 ? (many ? tdk_kv_append_rope_kernel<kMx4, true> : tdk_kv_append_rope_kernel<kMx4, false>)
                              : (many ? tdk_kv_append_rope_kernel<kBf16, true> : tdk_kv_append_rope_kernel<kBf16, false>);
  return launch(kernel, (int64_t)kv.n_tokens * rows.waves, 64, st, kv, rows);
}

}  // namespace tdk
