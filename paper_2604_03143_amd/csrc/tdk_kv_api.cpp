// Host side of the caches that programs append to: argument checks, how an attention call is cut, the C ABI.
// Everything the host can see is checked before the device is asked for, so every refusal can be had without a GPU.
#include <algorithm>
#include <cmath>
#include <limits>
#include <memory>

#include "tdk_errors.h"
#include "tdk_kv.h"
#include "tdk_plan.h"

using namespace tdk;

struct tdk_kv {
  tdk_model model{};
  int32_t   format = TDK_KV_BF16;
  int       device = -1;          // -1: created where no device is
  int32_t   n_cus = 256;
  double    inv_freq[kHalf];
};

namespace {

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;    // query rows of a call: their numbers are int32
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1; // of one launch
constexpr int32_t kMaxQHeads = 1 << 16;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;        // of a call, and of a sequence that a table has room for
constexpr float   kMaxScale = 0x1p127f;                  // times log2(e) still an fp32 number
constexpr int32_t kMaxSeqs = 1 << 30;                   // the search for a token's sequence counts in int32, in steps of 64

bool off(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// token strides of row buffers, in elements
bool bad_stride(int64_t stride, int64_t row) { return stride < row || (stride & 7) != 0 || stride > ((int64_t)1 << 40); }

tdk_status check_batch(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* b, bool* nothing) {
  if (!kv) return fail(TDK_ERR_INVALID_ARG, "kv handle is NULL");
  if (!cache || !b) return fail(TDK_ERR_INVALID_ARG, "cache / batch is NULL");
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_len < 0 || b->table_stride < 0) return fail(TDK_ERR_INVALID_ARG, "batch: negative size");
  if (cache->pool_pages < 0 || cache->pool_pages >= (int64_t)1 << 31) return fail(TDK_ERR_INVALID_ARG, "cache: pool_pages out of range");
  if (b->n_tokens > kMaxTokens || (int64_t)b->table_stride * kv->model.page_tokens > kMaxTokens)
    return fail(TDK_ERR_UNSUPPORTED, "batch: more than 2^30 tokens");
  if (b->n_seqs > kMaxSeqs) return fail(TDK_ERR_UNSUPPORTED, "batch: more than 2^30 sequences");
  *nothing = b->n_seqs == 0 || b->n_tokens == 0;
  if (*nothing) return TDK_OK;
  if (!b->q_start || !b->seq_len) return fail(TDK_ERR_INVALID_ARG, "batch: q_start / seq_len is NULL");
  if (b->table_stride > 0 && !b->block_table) return fail(TDK_ERR_INVALID_ARG, "batch: block_table is NULL");
  if (off(b->q_start, 4) || off(b->seq_len, 4) || off(b->block_table, 4)) return fail(TDK_ERR_INVALID_ARG, "batch: arrays must be 4-byte aligned");
  if (cache->pool_pages > 0 && (!cache->k || !cache->v)) return fail(TDK_ERR_INVALID_ARG, "cache holds a NULL plane");
  if (off(cache->k, 16) || off(cache->v, 16)) return fail(TDK_ERR_INVALID_ARG, "cache planes must be 16-byte aligned");
  return TDK_OK;
}

// last of all: the arguments are right, is this the handle's device?
tdk_status check_device(const tdk_kv* kv) {
  int dev = -1;
  if (kv->device < 0 || hipGetDevice(&dev) != hipSuccess || dev != kv->device)
    return fail(TDK_ERR_INVALID_ARG, "the handle was created on another device than the current one");
  return TDK_OK;
}

KvDev kv_dev(const tdk_kv* kv, const tdk_kv_cache* c, const tdk_kv_batch* b) {
  KvDev d;
  d.k = static_cast<char*>(c->k);
  d.v = static_cast<char*>(c->v);
  d.pool_pages = (int32_t)c->pool_pages;
  d.q_start = b->q_start;
  d.seq_len = b->seq_len;
  d.table = b->block_table;
  d.table_stride = b->table_stride;
  d.n_seqs = b->n_seqs;
  d.n_tokens = b->n_tokens;
  d.heads = kv->model.num_kv_heads;
  d.page_shift = kv->model.page_tokens == 32 ? 5 : 4;
  d.interleaved = kv->model.rope_style == TDK_ROPE_INTERLEAVED;
  return d;
}

tdk_status check_rows(const tdk_kv* kv, const tdk_kv_rows* r, bool reading) {
  const int64_t hd = (int64_t)kv->model.num_kv_heads * kHeadDim;
  if (!r->k || !r->v) return fail(TDK_ERR_INVALID_ARG, "rows: k / v is NULL");
  if (off(r->k, 16) || off(r->v, 16)) return fail(TDK_ERR_INVALID_ARG, "rows: k / v must be 16-byte aligned");
  if (bad_stride(r->k_stride, hd) || bad_stride(r->v_stride, hd))
    return fail(TDK_ERR_INVALID_ARG, "rows: strides must be multiples of 8, at least num_kv_heads * 128");
  if (reading) {
    if (r->q || r->q_out) return fail(TDK_ERR_INVALID_ARG, "rows: a cache holds no queries");
    return TDK_OK;
  }
  if (!r->q && !r->q_out) return TDK_OK;
  if (!r->q || !r->q_out) return fail(TDK_ERR_INVALID_ARG, "rows: q and q_out come together");
  if (r->n_q_heads < 1 || r->n_q_heads > kMaxQHeads) return fail(TDK_ERR_INVALID_ARG, "rows: n_q_heads out of range");
  if (off(r->q, 16) || off(r->q_out, 16)) return fail(TDK_ERR_INVALID_ARG, "rows: q / q_out must be 16-byte aligned");
  const int64_t qd = (int64_t)r->n_q_heads * kHeadDim;
  if (bad_stride(r->q_stride, qd) || bad_stride(r->q_out_stride, qd))
    return fail(TDK_ERR_INVALID_ARG, "rows: strides must be multiples of 8, at least n_q_heads * 128");
  if (r->q == r->q_out && r->q_stride != r->q_out_stride) return fail(TDK_ERR_INVALID_ARG, "rows: queries rotated in place keep their stride");
  return TDK_OK;
}

tdk_status move_rows(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch, const tdk_kv_rows* rows, bool reading,
                     void* hip_stream) {
  bool nothing = false;
  tdk_status st = check_batch(kv, cache, batch, &nothing);
  if (st != TDK_OK) return st;
  if (!rows) return fail(TDK_ERR_INVALID_ARG, "rows is NULL");
  if (!nothing && (st = check_rows(kv, rows, reading)) != TDK_OK) return st;
  KvRowsDev r{};
  r.k = static_cast<char*>(rows->k);
  r.v = static_cast<char*>(rows->v);
  r.k_stride = 2 * rows->k_stride;
  r.v_stride = 2 * rows->v_stride;
  if (rows->q) {
    r.q = static_cast<const char*>(rows->q);
    r.q_out = static_cast<char*>(rows->q_out);
    r.q_stride = 2 * rows->q_stride;
    r.q_out_stride = 2 * rows->q_out_stride;
    r.n_q_heads = rows->n_q_heads;
  }
  // A wavefront takes eight heads of a token at a time.  Few tokens: a workgroup for each eight heads, so that all of a call's
  // accesses are under way at once; many: the token's place and angles are found out once for all its heads.
  const int steps = (2 * kv->model.num_kv_heads + r.n_q_heads + 7) / 8;
  const bool many = (int64_t)batch->n_tokens * steps > (int64_t)8 * kv->n_cus;
  r.waves = many ? 1 : steps;
  if ((int64_t)batch->n_tokens * r.waves * 256 > kMaxThreads) return fail(TDK_ERR_UNSUPPORTED, "batch: more tokens than a launch holds");
  std::copy(std::begin(kv->inv_freq), std::end(kv->inv_freq), std::begin(r.inv_freq));
  st = check_device(kv);
  if (st != TDK_OK || nothing) return st;
  const KvDev d = kv_dev(kv, cache, batch);
  const bool four = kv->format == TDK_KV_MXFP4;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = reading ? launch_kv_read(d, r, four, many, s) : launch_kv_append(d, r, four, many, s);
  return e == hipSuccess ? TDK_OK : hip_fail(e, reading ? "kernel launch (tdk_kv_read)" : "kernel launch (tdk_kv_append)");
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Into how many parts each sequence is cut, at most (256 tokens a part at least).
//   Up to 128 rows per sequence (decoding, drafted tokens): a launch goes round by round, `resident` workgroups at a time (two per compute unit,
//   three of the 4-bit rows kernel), each as long as a part and what a part costs besides: its workgroup's start and its rows' partial results on
//   their way to memory and back, here in tokens.  The last round ends late on some compute units, a tenth of a round; so
//   many parts pay where there are few rounds (64 sequences of 16 000 tokens, one round 725 us, four 680; 66 of 4000 with 20 rows,
//   one part 275, six 237), and not where there are many (250 of 4000: one part 512, two 529).
//   More (prompts): only as many as fill the device; the blocks differ in length by themselves, and a part's rows are
//   many (four prompts of up to 2048 tokens: one part 523 us, two 662).
int64_t attend_parts(const tdk_kv* kv, int64_t blocks, int64_t len, int64_t per_seq, int block_rows) {
  const bool four = kv->format == TDK_KV_MXFP4;
  const int64_t resident = (four && block_rows == 16 ? 3 : 2) * (int64_t)kv->n_cus;
  const int64_t most = std::min<int64_t>((len + 255) / 256, 256);
  if (per_seq > 128 || blocks >= 16 * resident) return std::max<int64_t>(1, std::min((resident + blocks - 1) / blocks, most));
  const double extra = four ? 360 + 8.0 * per_seq : 120 + 2.0 * per_seq;
  int64_t best = 1;
  double least = INFINITY;
  for (int64_t c = 1; c <= most; ++c) {
    const int64_t rounds = (blocks * c + resident - 1) / resident;
    const double cost = rounds * ((double)len / c + (c > 1 ? extra : 0.0)) * (1.0 + 0.1 / rounds);
    if (cost < least) { least = cost; best = c; }
    if (rounds > 16) break;
  }
  return best;
}

// window, n_sink: as in the call; without a window the plan is the one with the most parts.  false: bad arguments
bool attend_plan_kv(const tdk_kv* kv, const tdk_kv_batch* b, int32_t n_q_heads, int32_t window, int32_t n_sink, KvAttendPlan& p) {
  const int32_t H = kv->model.num_kv_heads;
  if (b->n_seqs < 0 || b->n_tokens < 0 || b->max_len < 0 || n_q_heads < 1 || n_q_heads % H || n_q_heads > kMaxQHeads) return false;
  p = KvAttendPlan{};
  p.rows = (int64_t)b->n_tokens * n_q_heads;
  if (b->n_seqs == 0 || b->n_tokens == 0) return true;
  const int64_t group = n_q_heads / H;
  const int64_t per_seq = ((int64_t)b->n_tokens * group + b->n_seqs - 1) / b->n_seqs;      // rows of a sequence and KV head, on average
  // (sequences that differ in their new tokens: one token more than the average, so that fewer of them take several blocks; 64 of 4000 tokens,
  // up to 6 new ones, 5 heads per KV head: 215 -> 147 us, in 4 bits 74 -> 51)
  const int64_t rows = b->n_tokens > b->n_seqs && b->n_tokens % b->n_seqs ? per_seq + group : per_seq;
  // Rows per workgroup.  Up to 16: the rows kernel, which reads K straight into its products.  More: the step kernel, whose 128 rows meet tiles
  // in LDS; a few of its rows already read at the memory's rate in bf16 (64 sequences of 4000 tokens, 20 rows: 200 us, two passes of 16 rows
  // over the pages 290).  In 4 bits its tiles come by way of registers, one step ahead of another, and the rows kernel with 32 rows is ahead
  // up to two blocks (20 rows 61 us against 165; 64 rows 130 against 150; few sequences with 40 to 50 rows are up to 12 % behind).
  p.block_rows = rows <= 16 ? 16 : rows <= 64 && kv->format == TDK_KV_MXFP4 ? 32 : 128;
  p.forward = per_seq <= p.block_rows;
  p.ids = (int64_t)b->n_tokens * group / p.block_rows + b->n_seqs;
  // tokens that a block sees: all, or the window of its rows and the first tokens
  const int64_t seen = window > 0 ? std::min<int64_t>(b->max_len, (int64_t)window + n_sink + std::min<int64_t>(p.block_rows / group, b->n_tokens)) : b->max_len;
  const int64_t len = std::max<int64_t>(1, seen);
  const int64_t blocks = (per_seq + p.block_rows - 1) / p.block_rows * b->n_seqs * H;
  p.n_chunks = (int32_t)attend_parts(kv, blocks, len, per_seq, p.block_rows);
  const int64_t tile = p.block_rows == 128 ? 64 : 32;
  p.piece_tiles = (int32_t)(((len + tile - 1) / tile + p.n_chunks - 1) / p.n_chunks);
  if (p.n_chunks > 1) {
    p.o_part_ml = up256((size_t)p.rows * p.n_chunks * kHeadDim * sizeof(float));
    p.bytes = p.o_part_ml + up256((size_t)p.rows * p.n_chunks * 2 * sizeof(float));
  }
  return true;
}

}  // namespace

extern "C" {

tdk_status tdk_kv_create(const tdk_model* model, int32_t format, tdk_kv** out) {
  return guarded([&]() -> tdk_status {
    if (!out) return fail(TDK_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    std::string err;
    const tdk_status st = plan_check_model(model, err);
    if (st != TDK_OK) return fail(st, err);
    if (format != TDK_KV_BF16 && format != TDK_KV_MXFP4) return fail(TDK_ERR_UNSUPPORTED, "unknown cache format");
    auto kv = std::make_unique<tdk_kv>();
    kv->model = *model;
    kv->format = format;
    for (int j = 0; j < kHalf; ++j) kv->inv_freq[j] = std::pow(model->rope_theta, -(double)(2 * j) / (double)kHeadDim);
    int dev = -1, cus = 0;
    if (hipGetDevice(&dev) == hipSuccess) {
      kv->device = dev;
      if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && cus > 0) kv->n_cus = cus;
    } else {
      (void)hipGetLastError();
    }
    *out = kv.release();
    return TDK_OK;
  });
}

void tdk_kv_destroy(tdk_kv* kv) { delete kv; }

size_t tdk_kv_page_bytes(const tdk_kv* kv) {
  if (!kv) return 0;
  return (size_t)kv->model.page_tokens * kv->model.num_kv_heads * (kv->format == TDK_KV_MXFP4 ? 68 : 256);
}

tdk_status tdk_kv_append(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch, const tdk_kv_rows* rows, void* hip_stream) {
  return guarded([&] { return move_rows(kv, cache, batch, rows, false, hip_stream); });
}

tdk_status tdk_kv_read(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch, const tdk_kv_rows* rows, void* hip_stream) {
  return guarded([&] { return move_rows(kv, cache, batch, rows, true, hip_stream); });
}

size_t tdk_kv_attend_workspace_bytes(const tdk_kv* kv, const tdk_kv_batch* batch, int32_t n_q_heads) {
  KvAttendPlan p;
  return kv && batch && attend_plan_kv(kv, batch, n_q_heads, 0, 0, p) ? p.bytes : 0;
}

tdk_status tdk_kv_attend(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch, const tdk_kv_attend_io* a, void* hip_stream) {
  return guarded([&]() -> tdk_status {
    bool nothing = false;
    tdk_status st = check_batch(kv, cache, batch, &nothing);
    if (st != TDK_OK) return st;
    if (!a) return fail(TDK_ERR_INVALID_ARG, "attend io is NULL");
    KvAttendPlan p;
    if (!std::isfinite(a->scale)) return fail(TDK_ERR_INVALID_ARG, "scale must be finite");
    if (std::fabs(a->scale) > kMaxScale) return fail(TDK_ERR_INVALID_ARG, "scale: a magnitude above 2^127");
    if (a->window < 0 || a->n_sink < 0) return fail(TDK_ERR_INVALID_ARG, "window / n_sink is negative");
    if (!attend_plan_kv(kv, batch, a->n_q_heads, a->window, a->n_sink, p))
      return fail(TDK_ERR_INVALID_ARG, "n_q_heads must be a positive multiple of the KV heads");
    if (!a->part_out != !a->part_lse) return fail(TDK_ERR_INVALID_ARG, "part_out and part_lse come together");
    if (off(a->part_out, 16) || off(a->part_lse, 4) || off(a->hole, 4) || off(a->lse, 4))
      return fail(TDK_ERR_INVALID_ARG, "attend io: part_out must be 16-byte aligned, part_lse, hole and lse 4-byte");
    if (!nothing) {
      if (!a->q || !a->out) return fail(TDK_ERR_INVALID_ARG, "attend io holds a NULL buffer");
      if (off(a->q, 16) || off(a->out, 16)) return fail(TDK_ERR_INVALID_ARG, "q / out must be 16-byte aligned");
      const int64_t qd = (int64_t)a->n_q_heads * kHeadDim;
      if (bad_stride(a->q_stride, qd) || bad_stride(a->out_stride, qd))
        return fail(TDK_ERR_INVALID_ARG, "attend io: strides must be multiples of 8, at least n_q_heads * 128");
      if (p.bytes && !a->workspace) return fail(TDK_ERR_INVALID_ARG, "workspace is NULL");
      if (p.bytes && off(a->workspace, 256)) return fail(TDK_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
      if (a->workspace_bytes < p.bytes) return fail(TDK_ERR_INVALID_ARG, "workspace smaller than tdk_kv_attend_workspace_bytes()");
      if ((p.ids * p.n_chunks + 8) * kv->model.num_kv_heads * 256 > kMaxThreads || p.rows > kMaxRows)
        return fail(TDK_ERR_UNSUPPORTED, "attention launch larger than a grid");
    }
    st = check_device(kv);
    if (st != TDK_OK || nothing) return st;
    KvAttendDev at;
    at.q = static_cast<const char*>(a->q);
    at.out = static_cast<char*>(a->out);
    at.lse = a->lse;
    at.part_o = static_cast<float*>(a->workspace);
    at.part_ml = reinterpret_cast<float*>(static_cast<char*>(a->workspace) + p.o_part_ml);
    at.hole = a->hole;
    at.other_out = a->part_out;
    at.other_lse = a->part_lse;
    at.q_stride = 2 * a->q_stride;
    at.out_stride = 2 * a->out_stride;
    at.n_q_heads = a->n_q_heads;
    at.group = a->n_q_heads / kv->model.num_kv_heads;
    at.window = a->window;
    at.n_sink = a->n_sink;
    at.n_chunks = p.n_chunks;
    at.piece_tiles = p.piece_tiles;
    at.n_rest = (int32_t)(p.ids * p.n_chunks);
    at.q_flip = std::signbit(a->scale) ? 1 : 0;
    // (Zero, uniform weights, becomes the least number above it: what a row does not see stays minus infinity, and the scaled differences of all
    // other scores are below 2^-20.)
    at.scale = std::fmax(std::fabs(a->scale), std::numeric_limits<float>::denorm_min());
    at.scale2 = at.scale * 1.4426950408889634f;
    const hipError_t e = launch_kv_attend(kv_dev(kv, cache, batch), at, p, kv->format == TDK_KV_MXFP4, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? TDK_OK : hip_fail(e, "kernel launch (tdk_kv_attend)");
  });
}

}  // extern "C"
