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
  int       fmt = kBf16;          // as the kernels have it: kBf16, kMx4, kMx8
  int       device = -1;          // -1: created where no device is
  int32_t   n_cus = 256;
  int32_t   rotary = kHeadDim;
  double    magnitude = 1.0;
  double    inv_freq[kHalf];
};

namespace {

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;    // query rows of a call: their numbers are int32
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1; // of one launch
constexpr int32_t kMaxQHeads = 1 << 16;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;        // of a call, and of a sequence that a table has room for
constexpr float   kMaxScale = 0x1p127f;                  // times log2(e) still an fp32 number
constexpr int64_t kMaxKeyStride = (int64_t)1 << 24;     // elements: places in a step's tile of rows are 32-bit numbers of bytes
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

// Few tokens: a workgroup for each eight heads, so that all of a call's accesses are under way at once; many: the token's place and angles are
// found out once for all its heads.
int rows_steps(int heads) { return (heads + 7) / 8; }
bool many_rows(const tdk_kv* kv, const tdk_kv_batch* b, int steps) { return (int64_t)b->n_tokens * steps > (int64_t)8 * kv->n_cus; }

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
  const int steps = rows_steps(2 * kv->model.num_kv_heads + r.n_q_heads);
  const bool many = many_rows(kv, batch, steps);
  r.waves = many ? 1 : steps;
  if ((int64_t)batch->n_tokens * r.waves * 256 > kMaxThreads) return fail(TDK_ERR_UNSUPPORTED, "batch: more tokens than a launch holds");
  std::copy(std::begin(kv->inv_freq), std::end(kv->inv_freq), std::begin(r.inv_freq));
  r.rotary = kv->rotary;
  r.magnitude = kv->magnitude;
  st = check_device(kv);
  if (st != TDK_OK || nothing) return st;
  const KvDev d = kv_dev(kv, cache, batch);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = reading ? launch_kv_read(d, r, kv->fmt, many, s) : launch_kv_append(d, r, kv->fmt, many, s);
  return e == hipSuccess ? TDK_OK : hip_fail(e, reading ? "kernel launch (tdk_kv_read)" : "kernel launch (tdk_kv_append)");
}

// a plane of rows that are rotated: source and destination
tdk_status check_rotated(const void* x, int64_t stride, const void* out, int64_t out_stride, int64_t row, const char* what) {
  const std::string name(what);
  if (!x != !out) return fail(TDK_ERR_INVALID_ARG, "rotate io: " + name + " and " + name + "_out come together");
  if (!x) return TDK_OK;
  if (off(x, 16) || off(out, 16)) return fail(TDK_ERR_INVALID_ARG, "rotate io: " + name + " / " + name + "_out must be 16-byte aligned");
  if (bad_stride(stride, row) || bad_stride(out_stride, row))
    return fail(TDK_ERR_INVALID_ARG, "rotate io: strides must be multiples of 8, at least the heads * 128");
  if (x == out && stride != out_stride) return fail(TDK_ERR_INVALID_ARG, "rotate io: rows rotated in place keep their stride");
  return TDK_OK;
}

tdk_status rotate_rows(const tdk_kv* kv, const tdk_kv_batch* b, const tdk_kv_rotate_io* a, void* hip_stream) {
  if (!kv) return fail(TDK_ERR_INVALID_ARG, "kv handle is NULL");
  if (!b || !a) return fail(TDK_ERR_INVALID_ARG, "batch / rotate io is NULL");
  if (b->n_seqs < 0 || b->n_tokens < 0) return fail(TDK_ERR_INVALID_ARG, "batch: negative size");
  if (b->n_tokens > kMaxTokens) return fail(TDK_ERR_UNSUPPORTED, "batch: more than 2^30 tokens");
  if (b->n_seqs > kMaxSeqs) return fail(TDK_ERR_UNSUPPORTED, "batch: more than 2^30 sequences");
  if (a->q && (a->n_q_heads < 1 || a->n_q_heads > kMaxQHeads)) return fail(TDK_ERR_INVALID_ARG, "rotate io: n_q_heads out of range");
  tdk_status st = check_rotated(a->k, a->k_stride, a->k_out, a->k_out_stride, (int64_t)kv->model.num_kv_heads * kHeadDim, "k");
  if (st == TDK_OK) st = check_rotated(a->q, a->q_stride, a->q_out, a->q_out_stride, (int64_t)a->n_q_heads * kHeadDim, "q");
  if (st != TDK_OK) return st;
  const bool nothing = b->n_seqs == 0 || b->n_tokens == 0 || (!a->k && !a->q);
  if (!nothing && (!b->q_start || !b->seq_len)) return fail(TDK_ERR_INVALID_ARG, "batch: q_start / seq_len is NULL");
  if (off(b->q_start, 4) || off(b->seq_len, 4)) return fail(TDK_ERR_INVALID_ARG, "batch: arrays must be 4-byte aligned");
  KvRotateDev r{};
  if (a->k) {
    r.k = static_cast<const char*>(a->k);
    r.k_out = static_cast<char*>(a->k_out);
    r.k_stride = 2 * a->k_stride;
    r.k_out_stride = 2 * a->k_out_stride;
    r.n_k_heads = kv->model.num_kv_heads;
  }
  if (a->q) {
    r.q = static_cast<const char*>(a->q);
    r.q_out = static_cast<char*>(a->q_out);
    r.q_stride = 2 * a->q_stride;
    r.q_out_stride = 2 * a->q_out_stride;
    r.n_q_heads = a->n_q_heads;
  }
  const int steps = rows_steps(r.n_k_heads + r.n_q_heads);
  const bool many = many_rows(kv, b, steps);
  r.waves = many ? std::max(1, std::min(steps, 4)) : steps;
  if ((int64_t)b->n_tokens * 256 > kMaxThreads) return fail(TDK_ERR_UNSUPPORTED, "batch: more tokens than a launch holds");      // (four wavefronts a token at most where there are many)
  r.rotary = kv->rotary;
  r.cos_size = a->back ? 1.0 / kv->magnitude : kv->magnitude;
  r.sin_size = a->back ? -r.cos_size : r.cos_size;
  std::copy(std::begin(kv->inv_freq), std::end(kv->inv_freq), std::begin(r.inv_freq));
  st = check_device(kv);
  if (st != TDK_OK || nothing) return st;
  KvDev d{};
  d.q_start = b->q_start;
  d.seq_len = b->seq_len;
  d.n_seqs = b->n_seqs;
  d.n_tokens = b->n_tokens;
  d.page_shift = 4;
  d.interleaved = kv->model.rope_style == TDK_ROPE_INTERLEAVED;
  const hipError_t e = launch_kv_rotate(d, r, many, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? TDK_OK : hip_fail(e, "kernel launch (tdk_kv_rotate)");
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Into how many parts each sequence is cut, at most (256 tokens a part at least).
//   Up to 128 rows per sequence (decoding, drafted tokens): a launch goes round by round, `resident` workgroups at a time (two per compute unit,
//   three of the 4-bit rows kernel), each as long as a part and what a part costs besides: its workgroup's start and its rows' partial results on
//   their way to memory and back, here in tokens.  The last round ends late on some compute units, a tenth of a round; so
//   many parts pay where there are few rounds (64 sequences of 16 000 tokens, one round 725 us, four 680; 66 of 4000 with 20 rows,
//   one part 275, six 237), and not where there are many (250 of 4000: one part 512, two 529).
//   8 bits: the launch that joins the parts counts as well, as 300 tokens (100 sequences of 2000 tokens, three parts 82 us, one 68; 64 of 16 000, one part
//   315, five 297).
//   More (prompts): only as many as fill the device; the blocks differ in length by themselves, and a part's rows are
//   many (four prompts of up to 2048 tokens: one part 523 us, two 662).
int64_t attend_parts(int64_t resident, int fmt, int64_t blocks, int64_t len, int64_t per_seq) {
  const int64_t most = std::min<int64_t>((len + 255) / 256, 256);
  if (per_seq > 128 || blocks >= 16 * resident) return std::max<int64_t>(1, std::min((resident + blocks - 1) / blocks, most));
  const double extra = fmt == kMx4 ? 360 + 8.0 * per_seq : fmt == kMx8 ? 110 + 4.0 * per_seq : 120 + 2.0 * per_seq, join = fmt == kMx8 ? 300 : 0;
  int64_t best = 1;
  double least = INFINITY;
  for (int64_t c = 1; c <= most; ++c) {
    const int64_t rounds = (blocks * c + resident - 1) / resident;
    const double cost = rounds * ((double)len / c + (c > 1 ? extra : 0.0)) * (1.0 + 0.1 / rounds) + (c > 1 ? join : 0.0);
    if (cost < least) { least = cost; best = c; }
    if (rounds > 16) break;
  }
  return best;
}

tdk_status kv_create(const tdk_model* model, const tdk_rope* rope, int32_t format, tdk_kv** out) {
  if (!out) return fail(TDK_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  std::string err;
  tdk_status st = plan_check_model(model, err);
  if (st == TDK_OK && rope) st = plan_check_rope(model, rope, err);
  if (st != TDK_OK) return fail(st, err);
  if (format != TDK_KV_BF16 && format != TDK_KV_MXFP4 && format != TDK_KV_MXFP8) return fail(TDK_ERR_UNSUPPORTED, "unknown cache format");
  auto kv = std::make_unique<tdk_kv>();
  kv->model = *model;
  kv->fmt = format == TDK_KV_MXFP8 ? kMx8 : format == TDK_KV_MXFP4 ? kMx4 : kBf16;
  rope_frequencies(model, rope, kv->inv_freq);
  if (rope) {
    kv->rotary = rope->rotary_dim;
    kv->magnitude = rope->magnitude;
  }
  int dev = -1, cus = 0;
  if (hipGetDevice(&dev) == hipSuccess) {
    kv->device = dev;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && cus > 0) kv->n_cus = cus;
  } else {
    (void)hipGetLastError();
  }
  *out = kv.release();
  return TDK_OK;
}

void plan_space(KvAttendPlan& p) {
  if (p.n_chunks <= 1) return;
  p.o_part_ml = up256((size_t)p.rows * p.n_chunks * kHeadDim * sizeof(float));
  p.bytes = p.o_part_ml + up256((size_t)p.rows * p.n_chunks * 2 * sizeof(float));
}

// what both kinds of attention take besides their rows
struct Shared {
  const void* q;
  int64_t q_stride;
  int32_t n_q_heads;
  float scale;
  const void* out;
  int64_t out_stride;
  const float* lse;
  const void* workspace;
  size_t workspace_bytes;
  int32_t window, n_sink;
  const float *part_out, *part_lse;
};

tdk_status check_attend(const Shared& a, bool planned) {
  if (!std::isfinite(a.scale)) return fail(TDK_ERR_INVALID_ARG, "scale must be finite");
  if (std::fabs(a.scale) > kMaxScale) return fail(TDK_ERR_INVALID_ARG, "scale: a magnitude above 2^127");
  if (a.window < 0 || a.n_sink < 0) return fail(TDK_ERR_INVALID_ARG, "window / n_sink is negative");
  if (!planned) return fail(TDK_ERR_INVALID_ARG, "n_q_heads must be a positive multiple of the KV heads");
  if (!a.part_out != !a.part_lse) return fail(TDK_ERR_INVALID_ARG, "part_out and part_lse come together");
  return TDK_OK;
}
tdk_status check_attend_buffers(const Shared& a, const KvAttendPlan& p, int32_t heads) {
  if (!a.q || !a.out) return fail(TDK_ERR_INVALID_ARG, "attend io holds a NULL buffer");
  if (off(a.q, 16) || off(a.out, 16)) return fail(TDK_ERR_INVALID_ARG, "q / out must be 16-byte aligned");
  const int64_t qd = (int64_t)a.n_q_heads * kHeadDim;
  if (bad_stride(a.q_stride, qd) || bad_stride(a.out_stride, qd))
    return fail(TDK_ERR_INVALID_ARG, "attend io: strides must be multiples of 8, at least n_q_heads * 128");
  if (p.bytes && !a.workspace) return fail(TDK_ERR_INVALID_ARG, "workspace is NULL");
  if (p.bytes && off(a.workspace, 256)) return fail(TDK_ERR_INVALID_ARG, "the workspace must be 256-byte aligned");
  if (a.workspace_bytes < p.bytes) return fail(TDK_ERR_INVALID_ARG, "workspace smaller than the call's workspace_bytes()");
  if ((p.ids * p.n_chunks + 8) * heads * 256 > kMaxThreads || p.rows > kMaxRows)
    return fail(TDK_ERR_UNSUPPORTED, "attention launch larger than a grid");
  return TDK_OK;
}
void attend_dev(const tdk_kv* kv, const Shared& a, const KvAttendPlan& p, KvAttendDev& at) {
  at.q = static_cast<const char*>(a.q);
  at.out = static_cast<char*>(const_cast<void*>(a.out));
  at.lse = const_cast<float*>(a.lse);
  at.part_o = static_cast<float*>(const_cast<void*>(a.workspace));
  at.part_ml = reinterpret_cast<float*>(static_cast<char*>(const_cast<void*>(a.workspace)) + p.o_part_ml);
  at.hole = nullptr;
  at.other_out = a.part_out;
  at.other_lse = a.part_lse;
  at.q_stride = 2 * a.q_stride;
  at.out_stride = 2 * a.out_stride;
  at.n_q_heads = a.n_q_heads;
  at.group = a.n_q_heads / kv->model.num_kv_heads;
  at.group_inv = (uint32_t)(((1u << 22) + at.group - 1) / at.group);
  at.window = a.window;
  at.n_sink = a.n_sink;
  at.n_chunks = p.n_chunks;
  at.piece_tiles = p.piece_tiles;
  at.n_rest = (int32_t)(p.ids * p.n_chunks);
  at.q_flip = std::signbit(a.scale) ? 1 : 0;
  // (Zero, uniform weights, becomes the least number above it: what a row does not see stays minus infinity, and the scaled differences of all
  // other scores are below 2^-20.)
  at.scale = std::fmax(std::fabs(a.scale), std::numeric_limits<float>::denorm_min());
  at.scale2 = at.scale * 1.4426950408889634f;
}

// window, n_sink: as in the call; without a window the plan is the one with the most parts (attend_parts' cost of c parts is a(c) len + b(c), and
// b never falls with c: a shorter length never gains from more).  false: bad arguments
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
  // up to two blocks (20 rows 61 us against 165; 64 rows 130 against 150; few sequences with 40 to 50 rows are up to 12 % behind).  In 8 bits for one
  // block (20 rows 88 us against 109; 40 rows 172 against 118, 64 rows 186 against 120).
  p.block_rows = rows <= 16 ? 16 : rows <= (kv->fmt == kMx4 ? 64 : kv->fmt == kMx8 ? 32 : 0) ? 32 : 128;
  p.forward = per_seq <= p.block_rows;
  p.ids = (int64_t)b->n_tokens * group / p.block_rows + b->n_seqs;
  // tokens that a block sees: all, or the window of its rows and the first tokens
  const int64_t seen = window > 0 ? std::min<int64_t>(b->max_len, (int64_t)window + n_sink + std::min<int64_t>(p.block_rows / group, b->n_tokens)) : b->max_len;
  const int64_t len = std::max<int64_t>(1, seen);
  const int64_t blocks = (per_seq + p.block_rows - 1) / p.block_rows * b->n_seqs * H;
  p.n_chunks = (int32_t)attend_parts((kv->fmt == kMx4 && p.block_rows == 16 ? 3 : 2) * (int64_t)kv->n_cus, kv->fmt, blocks, len, per_seq);
  const int64_t tile = p.block_rows == 128 ? 64 : 32;
  p.piece_tiles = (int32_t)(((len + tile - 1) / tile + p.n_chunks - 1) / p.n_chunks);
  plan_space(p);
  return true;
}

// Parts of a prompt's keys: what a call takes in us with each number of them.  A workgroup's step takes 1.1 alone on its compute unit, 2 beside
// another; its start and end 6; the parts' results go to memory and back at 4 TB/s, in a launch of their own.
int64_t prompt_parts(int64_t n_cus, int64_t blocks, int64_t steps, int64_t rows) {
  const int64_t most = std::min<int64_t>((steps + 3) / 4, 256);
  int64_t best = 1;
  double least = INFINITY;
  for (int64_t c = 1; c <= most; ++c) {
    const int64_t groups = blocks * c, rounds = (groups + 2 * n_cus - 1) / (2 * n_cus);
    const double cost = rounds * ((groups <= n_cus ? 1.1 : 2.0) * ((steps + c - 1) / c) + 6.0) + (c > 1 ? 5.0 + rows * c * 1040.0 / 4e6 : 0.0);
    if (cost < least) { least = cost; best = c; }
    if (rounds > 2) break;
  }
  return best;
}

// The same for rows that are not in pages.  (A few queries behind long keys take these blocks as well, most of whose rows are then idle: 64 sequences of 4000 and 16 000
// keys, 8 heads with 5 queries, one token each 160 and 598 us, 4.8 and 5.3 TB/s, four tokens 163 and 615; 256 of 4000 551 us, 5.7 TB/s; four of 16 000 38 us, 5.3.)
bool prompt_plan(const tdk_kv* kv, const tdk_prompt_batch* b, int32_t n_q_heads, int32_t window, int32_t n_sink, KvAttendPlan& p) {
  const int32_t H = kv->model.num_kv_heads;
  if (b->n_seqs < 0 || b->n_q < 0 || b->n_k < 0 || b->max_len < 0 || n_q_heads < 1 || n_q_heads % H || n_q_heads > kMaxQHeads) return false;
  p = KvAttendPlan{};
  p.rows = (int64_t)b->n_q * n_q_heads;
  if (b->n_seqs == 0 || b->n_q == 0) return true;
  const int64_t group = n_q_heads / H;
  const int64_t per_seq = ((int64_t)b->n_q * group + b->n_seqs - 1) / b->n_seqs;      // rows of a sequence and KV head, on average
  p.block_rows = 128;
  p.forward = per_seq <= p.block_rows;
  p.ids = (int64_t)b->n_q * group / p.block_rows + b->n_seqs;
  const int64_t seen = window > 0 ? std::min<int64_t>(b->max_len, (int64_t)window + n_sink + std::min<int64_t>(p.block_rows / group, b->n_q)) : b->max_len;
  const auto steps_of = [](int64_t len) { return std::max<int64_t>(1, (len + 63) / 64); };
  const int64_t steps = steps_of(seen), blocks = (per_seq + p.block_rows - 1) / p.block_rows * b->n_seqs * H;
  p.n_chunks = (int32_t)prompt_parts(kv->n_cus, blocks, steps_of(b->max_len), p.rows);      // (the workspace has room for so many, whatever the window)
  if (seen < b->max_len) p.n_chunks = std::min(p.n_chunks, (int32_t)prompt_parts(kv->n_cus, blocks, steps, p.rows));
  p.piece_tiles = (int32_t)((steps + p.n_chunks - 1) / p.n_chunks);
  plan_space(p);
  return true;
}

}  // namespace

extern "C" {

tdk_status tdk_kv_create(const tdk_model* model, int32_t format, tdk_kv** out) {
  return guarded([&] { return kv_create(model, nullptr, format, out); });
}

tdk_status tdk_kv_create_rope(const tdk_model* model, const tdk_rope* rope, int32_t format, tdk_kv** out) {
  return guarded([&]() -> tdk_status {
    if (out) *out = nullptr;
    return rope ? kv_create(model, rope, format, out) : fail(TDK_ERR_INVALID_ARG, "rope is NULL");
  });
}

tdk_status tdk_kv_rotate(const tdk_kv* kv, const tdk_kv_batch* batch, const tdk_kv_rotate_io* io, void* hip_stream) {
  return guarded([&] { return rotate_rows(kv, batch, io, hip_stream); });
}

void tdk_kv_destroy(tdk_kv* kv) { delete kv; }

size_t tdk_kv_page_bytes(const tdk_kv* kv) {
  if (!kv) return 0;
  return (size_t)kv->model.page_tokens * kv->model.num_kv_heads * (kv->fmt == kMx4 ? 68 : kv->fmt == kMx8 ? 132 : 256);
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
    const Shared sh{a->q, a->q_stride, a->n_q_heads, a->scale, a->out, a->out_stride, a->lse, a->workspace, a->workspace_bytes,
                    a->window, a->n_sink, a->part_out, a->part_lse};
    st = check_attend(sh, attend_plan_kv(kv, batch, a->n_q_heads, std::max(a->window, 0), std::max(a->n_sink, 0), p));
    if (st != TDK_OK) return st;
    if (off(a->part_out, 16) || off(a->part_lse, 4) || off(a->hole, 4) || off(a->lse, 4))
      return fail(TDK_ERR_INVALID_ARG, "attend io: part_out must be 16-byte aligned, part_lse, hole and lse 4-byte");
    if (!nothing && (st = check_attend_buffers(sh, p, kv->model.num_kv_heads)) != TDK_OK) return st;
    st = check_device(kv);
    if (st != TDK_OK || nothing) return st;
    KvAttendDev at;
    attend_dev(kv, sh, p, at);
    at.hole = a->hole;
    at.last_id = p.forward ? -1 : (int32_t)(p.ids - 1);
    const hipError_t e = launch_kv_attend(kv_dev(kv, cache, batch), at, p, kv->fmt, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? TDK_OK : hip_fail(e, "kernel launch (tdk_kv_attend)");
  });
}

size_t tdk_prompt_attend_workspace_bytes(const tdk_kv* kv, const tdk_prompt_batch* batch, int32_t n_q_heads) {
  KvAttendPlan p;
  return kv && batch && prompt_plan(kv, batch, n_q_heads, 0, 0, p) ? p.bytes : 0;
}

tdk_status tdk_prompt_attend(const tdk_kv* kv, const tdk_prompt_batch* b, const tdk_prompt_attend_io* a, void* hip_stream) {
  return guarded([&]() -> tdk_status {
    if (!kv) return fail(TDK_ERR_INVALID_ARG, "kv handle is NULL");
    if (!b || !a) return fail(TDK_ERR_INVALID_ARG, "batch / attend io is NULL");
    if (b->n_seqs < 0 || b->n_q < 0 || b->n_k < 0 || b->max_len < 0) return fail(TDK_ERR_INVALID_ARG, "batch: negative size");
    if (b->n_q > kMaxTokens || b->n_k > kMaxTokens) return fail(TDK_ERR_UNSUPPORTED, "batch: more than 2^30 tokens");
    if (b->n_seqs > kMaxSeqs) return fail(TDK_ERR_UNSUPPORTED, "batch: more than 2^30 sequences");
    const bool nothing = b->n_seqs == 0 || b->n_q == 0;
    if (!nothing && (!b->q_start || !b->k_start)) return fail(TDK_ERR_INVALID_ARG, "batch: q_start / k_start is NULL");
    if (off(b->q_start, 4) || off(b->k_start, 4)) return fail(TDK_ERR_INVALID_ARG, "batch: arrays must be 4-byte aligned");
    KvAttendPlan p;
    const Shared sh{a->q, a->q_stride, a->n_q_heads, a->scale, a->out, a->out_stride, a->lse, a->workspace, a->workspace_bytes,
                    a->window, a->n_sink, a->part_out, a->part_lse};
    tdk_status st = check_attend(sh, prompt_plan(kv, b, a->n_q_heads, std::max(a->window, 0), std::max(a->n_sink, 0), p));
    if (st != TDK_OK) return st;
    if (off(a->part_out, 16) || off(a->part_lse, 4) || off(a->lse, 4))
      return fail(TDK_ERR_INVALID_ARG, "attend io: part_out must be 16-byte aligned, part_lse and lse 4-byte");
    if (!nothing) {
      if ((st = check_attend_buffers(sh, p, kv->model.num_kv_heads)) != TDK_OK) return st;
      const int64_t hd = (int64_t)kv->model.num_kv_heads * kHeadDim;
      if (b->n_k > 0 && (!a->k || !a->v)) return fail(TDK_ERR_INVALID_ARG, "attend io: k / v is NULL");
      if (off(a->k, 16) || off(a->v, 16)) return fail(TDK_ERR_INVALID_ARG, "k / v must be 16-byte aligned");
      if (bad_stride(a->k_stride, hd) || bad_stride(a->v_stride, hd) || a->k_stride > kMaxKeyStride || a->v_stride > kMaxKeyStride)
        return fail(TDK_ERR_INVALID_ARG, "attend io: k and v strides must be multiples of 8, at least num_kv_heads * 128 and at most 2^24");
    }
    st = check_device(kv);
    if (st != TDK_OK || nothing) return st;
    KvDev d{};
    d.k = static_cast<char*>(const_cast<void*>(a->k));
    d.v = static_cast<char*>(const_cast<void*>(a->v));
    d.q_start = b->q_start;
    d.n_seqs = b->n_seqs;
    d.n_tokens = b->n_q;
    d.heads = kv->model.num_kv_heads;
    PromptAttendDev at;
    attend_dev(kv, sh, p, at);
    at.k_start = b->k_start;
    at.k_stride = 2 * a->k_stride;
    at.v_stride = 2 * a->v_stride;
    at.n_k = b->n_k;
    at.f32 = a->out_f32 != 0;
    if (at.f32) at.out_stride *= 2;
    // Blocks of one length of rows (a block per sequence) as they come; else a causal prompt's last rows see most and start first.  One sequence whose
    // blocks all find room at once, two on a compute unit: the second half the other way round, so that long ones have short ones beside them (8192 tokens
    // and 8 heads with a query each: 181 -> 172 us).
    at.last_id = (int32_t)(p.ids - 1);
    at.down = p.forward ? 0 : (int32_t)p.ids;
    const int64_t full = (p.rows / d.heads + 127) / 128, room = kv->n_cus / d.heads;      // blocks of one sequence and KV head, compute units for them
    if (!p.forward && b->n_seqs == 1 && p.n_chunks == 1 && full <= 2 * room) at.down = (int32_t)std::min<int64_t>(p.ids, room + p.ids - full);
    const hipError_t e = launch_prompt_attend(d, at, p, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? TDK_OK : hip_fail(e, "kernel launch (tdk_prompt_attend)");
  });
}

}  // extern "C"
