/*
 * tdk.h -- C ABI of libtdk: the data-parallel hot path of collective KV-cache reuse and
 * diff-aware storage for multi-agent "All-Gather" rounds, for AMD MI355X (gfx950).
 *
 * One round = n_sessions masters (the K/V of the shared output blocks, cached once, rotated for
 * positions master_pos0 ..) and n_agents mirrors (agent sub-requests).  Every agent's prompt is its
 * private history followed by the shared blocks (Sec. 2.1, Eq. 2), so agent i sees the shared span
 * at absolute positions dst_pos0_i .. dst_pos0_i + S - 1.  Per layer the library offers three
 * collective steps over the whole round:
 *
 *   tdk_rerotate_round   Sec. 4.2 "Layerwise Collective Reuse": one batched RoPE pass for the
 *                        group; cached K re-rotated by the position delta, V copied.
 *   tdk_diff_encode      Sec. 4.3 "Block-Sparse Diff Representation", Sec. 5 "Diff-Aware Storage":
 *                        each mirror becomes {touched page indices, K/V values of those pages}.
 *   tdk_diff_decode      Sec. 4.4 / Algorithm 1 "Fused Diff Restore": apply diff, recover RoPE
 *                        positions, write through the slot map; no dense mirror is materialised.
 *
 * Conventions
 *   - Pointers marked DEV are device pointers owned by the caller; HOST are host pointers.  The
 *     library borrows DEV buffers for the duration of the enqueued work and never frees them.
 *   - The three step calls validate on the host, enqueue kernels on the given HIP stream
 *     (hipStream_t passed as void*, NULL = default stream) and return without synchronising.
 *     They allocate nothing.  tdk_round_create / tdk_round_destroy allocate / free the library's
 *     own device memory (tables, descriptors, per-page flag scratch) and are synchronous.
 *   - Errors are return codes; tdk_last_error() gives thread-local detail.  Anything the host can
 *     detect fails before any work is enqueued.  No exception leaves the library.  A round belongs to
 *     the device that was current when it was created; step calls made with another device current
 *     fail with INVALID_ARG.
 *   - Results are deterministic: same inputs, same bits, including index order and payload placement.
 *   - Not checked (preconditions): physical pages of different agents do not overlap (a precondition of
 *     grouping requests, Sec. 4.2); buffers are not written concurrently; calls on one
 *     round are issued in stream order on one stream at a time (encode uses the round's own flag
 *     scratch, restore its events), different rounds are independent.
 *
 * Arithmetic: bf16 storage; cos/sin of phi_j = delta * theta^(-2j/D) evaluated in double on the
 * host and rounded once to fp32; per pair (a, b): y_a = fma(x_a, cos, -(x_b * sin)),
 * y_b = fma(x_b, cos, x_a * sin) in fp32; round-to-nearest-even to bf16.
 */
#ifndef TDK_H
#define TDK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TDK_OK = 0,
  TDK_ERR_INVALID_ARG = 1,   /* NULL, out-of-range or inconsistent argument           */
  TDK_ERR_UNSUPPORTED = 2,   /* a valid request this build has no kernel for          */
  TDK_ERR_CAPACITY = 3,      /* the round exceeds a fixed limit of the call (tdk_diff_encode_static); a diff
                                buffer that is too small is reported on the device (tdk_diff.overflow)  */
  TDK_ERR_HIP = 4,           /* a HIP runtime call failed (no GPU, launch error, ...)  */
  TDK_ERR_NOMEM = 5          /* host or device allocation failed                      */
} tdk_status;

#define TDK_BF16 0
#define TDK_ROPE_HALF 0          /* pair (j, j + D/2) inside a head */
#define TDK_ROPE_INTERLEAVED 1   /* pair (2j, 2j + 1) inside a head */

const char* tdk_status_str(tdk_status s);   /* static string                                   */
const char* tdk_last_error(void);           /* thread-local, valid until the next failing call */
const char* tdk_version(void);

/* Cache geometry.  Supported: dtype TDK_BF16; head_dim 128; 1 <= num_kv_heads <= 8;
 * page_tokens 16 or 32; both rope styles. */
typedef struct {
  int32_t num_layers;
  int32_t num_kv_heads;   /* H */
  int32_t head_dim;       /* D */
  int32_t page_tokens;    /* T: tokens per page = granularity of the diff (Sec. 4.3) */
  int32_t dtype;          /* TDK_BF16 */
  int32_t rope_style;     /* TDK_ROPE_* */
  double  rope_theta;
} tdk_model;

/* How positions become angles beyond rope_theta alone.  A pair j < rotary_dim / 2 turns by f_j = theta^(-2 j / rotary_dim)
 * radians per position; the elements behind rotary_dim pass as they are (half layout: pairs (j, j + rotary_dim / 2),
 * interleaved: (2 j, 2 j + 1)).  For contexts `factor` times as long as the original_len tokens that a model was trained on:
 *   LINEAR   every frequency is divided by factor
 *   TURNS    by the turns r_j = original_len f_j / (2 pi) that a pair makes: those below `low` are divided by factor, those above
 *            `high` stay, between them the share (r_j - low) / (high - low) of f_j stays and the rest is divided
 *   INDEX    by the pair's number: with d(r) = rotary_dim ln(original_len / (2 pi r)) / (2 ln theta), the number of the pair that makes r
 *            turns, the divided share grows from 0 at a = max(floor d(high), 0) to 1 at b = min(ceil d(low), rotary_dim - 1); where b is
 *            not above a, the pairs up to a stay and those behind are divided
 * magnitude: cosines and sines are multiplied by it (in double, before they are rounded to fp32).  Fields that a scaling does not use are
 * not looked at.  Errors of the calls that take one: UNSUPPORTED (rotary_dim not a multiple of 16 from 16 to 128, unknown scaling),
 * INVALID_ARG (magnitude outside [1e-6, 1e6], factor below 1, original_len not positive, not 0 < low < high; INDEX with theta <= 1). */
#define TDK_ROPE_SCALE_NONE   0
#define TDK_ROPE_SCALE_LINEAR 1
#define TDK_ROPE_SCALE_TURNS  2
#define TDK_ROPE_SCALE_INDEX  3
typedef struct {
  int32_t rotary_dim;
  int32_t scaling;        /* TDK_ROPE_SCALE_* */
  double  factor;
  double  original_len;
  double  low;
  double  high;
  double  magnitude;
} tdk_rope;

/* One shared span = one master. */
typedef struct {
  int32_t span_tokens;    /* S >= 0 */
  int64_t master_pos0;    /* absolute position the master's token 0 is rotated for */
} tdk_session;

/* One run of consecutive master tokens in an agent's prompt: master tokens src_tok .. src_tok+len-1
 * land at absolute positions dst_pos .. dst_pos+len-1.  diff_pos is the position the run started at
 * when the diff that will be restored was encoded (the per-segment form of tdk_agent::diff_pos0):
 * equal to dst_pos for a diff of this round; otherwise the K values of the run's payload rows are
 * re-rotated by dst_pos - diff_pos on restore.  Ignored by encode. */
typedef struct {
  int32_t src_tok;
  int32_t len;
  int64_t dst_pos;
  int64_t diff_pos;
} tdk_segment;

/* One agent sub-request (a mirror of its session's master). */
typedef struct {
  int32_t        session;          /* index into sessions[]                                        */
  int64_t        dst_pos0;         /* absolute position of its first shared token (history length) */
  const int32_t* block_table;      /* HOST: logical page -> physical page of the agent's sequence  */
  int32_t        block_table_len;  /* >= ceil((dst_pos0 + S) / T)                                  */
  int64_t        diff_pos0;        /* position of its first shared token when the diff that will be
                                      given to tdk_diff_decode / tdk_restore_layers was encoded: equal
                                      to dst_pos0 for a diff of this round; for a mirror stored in an
                                      earlier round its K values are re-rotated by dst_pos0 - diff_pos0
                                      on restore (Alg. 1, RoPERecover(P_old, P_new)).  Ignored by encode. */
  int32_t        n_segments;       /* 0: identity layout (the shared span sits at dst_pos0 .. dst_pos0+S-1).
                                      > 0: the scheduler-defined layout of the shared blocks for this agent
                                      (Sec. 2.1, Eq. 2): segments sorted by src_tok, covering [0, S) exactly
                                      once, destinations disjoint, every master page meeting at most two
                                      segments (true whenever blocks are at least a page long); dst_pos0 and
                                      diff_pos0 are then unused (each segment carries its own diff_pos). */
  const tdk_segment* segments;     /* HOST */
} tdk_agent;

typedef struct tdk_round tdk_round;   /* opaque: tables, descriptors, scratch on the current device */

/* Builds the plan of a round on the current HIP device: rotation tables per agent, the slices of
 * the block tables that cover the shared spans, the work list.  Copies everything it needs; the
 * arguments may be freed on return.  Errors: INVALID_ARG (NULL, negative sizes or positions, bad
 * session index, block table too short, negative page number, position beyond 2^31), UNSUPPORTED
 * (geometry), NOMEM, HIP. */
tdk_status tdk_round_create(const tdk_model* model,
                            const tdk_session* sessions, int32_t n_sessions,
                            const tdk_agent* agents, int32_t n_agents,
                            tdk_round** out);
/* The same for caches whose keys were rotated by `rope` (tdk_kv_create_rope): re-rotation goes by its frequencies.  The cached keys carry the
 * magnitude already.  Whole heads only: rotary_dim other than 128 is UNSUPPORTED. */
tdk_status tdk_round_create_rope(const tdk_model* model, const tdk_rope* rope,
                                 const tdk_session* sessions, int32_t n_sessions,
                                 const tdk_agent* agents, int32_t n_agents,
                                 tdk_round** out);
void       tdk_round_destroy(tdk_round* r);             /* NULL-safe */
size_t     tdk_scratch_bytes(const tdk_round* r);       /* device bytes the round owns */

/* Launch shape and cache policy.  agents_per_group: agents of one session that share one read of a
 * master page (1..32), 0 = automatic.  flags: which accesses carry the non-temporal hint (streamed
 * through L2 and written back early instead of lingering as dirty lines that the next kernel has to
 * flush); the default was measured best for the whole rerotate / decode / encode sequence.
 * Synchronises the device (the work list it replaces may still be in use).  Results never depend on
 * these settings.  Work lists longer than the automatic ones (smaller groups, TDK_TUNE_TAPER) need device
 * memory of their own, once per round: 192 bytes per (agent, page) pair, else NOMEM.  Calls captured in a
 * graph keep the lengths of their time: capture them again after lists have become longer. */
#define TDK_TUNE_NT_REROTATE_STORES 1
#define TDK_TUNE_NT_DECODE_STORES   2
#define TDK_TUNE_NT_COMPARE_LOADS   4
#define TDK_TUNE_NT_SCATTER         8
#define TDK_TUNE_NT_GATHER          16
#define TDK_TUNE_PREFETCH_MASTER    32   /* rerotate: the first workgroups sweep the masters into the
                                            memory-side cache before anything is written           */
#define TDK_TUNE_PREFETCH_MASTER_DECODE 64 /* the same in decode: worth 5 % when its masters were not just
                                            read by another kernel, costs 0.6 % when they were    */
#define TDK_TUNE_XCD_QUEUES         128  /* the page kernels that write: two looping workgroups per compute unit take work
                                            items from one queue per XCD and, when theirs is empty, from the others' (the
                                            XCDs do not write at the same rate); off: one workgroup per item, fixed to an
                                            XCD by its number */
#define TDK_TUNE_TAPER              256  /* work list: smaller agent groups for the last pages, so that a launch does not
                                            end with a few long items on an otherwise idle chip                      */
#define TDK_TUNE_QUEUES_ANY_SIZE    512  /* queues also for rounds with fewer than four items per resident workgroup
                                            (by default such launches stay static: it is faster there)             */
#define TDK_TUNE_SCATTER_IN_DECODE  1024 /* small rounds (static launches): the workgroups that copy the listed pages ride
                                            behind the page items of decode's launch instead of a launch of their own */
#define TDK_TUNE_SHARED_TAIL        2048 /* static launches of the kernels that write: the last fifth of the work items goes
                                            to whichever of the launch's last workgroups start first (an XCD that writes
                                            faster takes more of it) instead of to fixed workgroups                     */
#define TDK_TUNE_ALL                4095
#define TDK_TUNE_DEFAULT            (191 + 1024 + 2048)
tdk_status tdk_round_tune(tdk_round* r, int32_t agents_per_group, int32_t flags);
int32_t    tdk_round_agents_per_group(const tdk_round* r);   /* the value in use (resolved if automatic); 0 for NULL */

/* Per-layer views, all DEV.
 *   master_k/v  [sum_s S_s][H][D] bf16, sessions concatenated in order (token-major rows)
 *   pool_k/v    [pool_pages][T][H][D] bf16, the paged KV memory of this layer */
typedef struct {
  const void* master_k;
  const void* master_v;
  void*       pool_k;
  void*       pool_v;
  int64_t     pool_pages;
} tdk_layer_io;

/* The mirrors of one layer (block-sparse diff of every agent), all DEV, caller-owned.
 *   count[n_agents]        pages in each agent's diff
 *   offset[n_agents + 1]   exclusive prefix of count
 *   idx[capacity_pages]    master-page numbers, ascending within an agent, agents in order
 *   payload[capacity_pages][2][T][H][D]  the agent's own K rows then V rows of each listed page
 *                          (values as they sit in the agent's cache; rows past the span are zero)
 *   overflow[1]            set to 1 by encode when sum(count) > capacity_pages, else 0; count and
 *                          offset are complete either way and nothing is written past capacity. */
typedef struct {
  int32_t* count;
  int64_t* offset;
  int32_t* idx;
  void*    payload;
  int64_t  capacity_pages;
  int32_t* overflow;
} tdk_diff;

/* pool_k[slot_i(m)] = bf16(R(dst_pos0_i - master_pos0) master_k[m]), pool_v[slot_i(m)] = master_v[m]
 * for every agent i and master token m, slot_i(m) = block_table_i[(dst_pos0_i+m)/T]*T + (dst_pos0_i+m)%T.
 * No other pool row is written.  Errors: INVALID_ARG (NULL, layer out of range, pool_pages smaller
 * than the largest mapped page + 1), HIP. */
tdk_status tdk_rerotate_round(tdk_round* r, int32_t layer, const tdk_layer_io* io, void* hip_stream);

/* Page p of agent i is in the diff iff some valid element of its K or V rows has
 * !(|a - ref| <= eps) in fp32, ref = what tdk_rerotate_round would write.  eps >= 0, not NaN.
 * Reads the pool, writes *out.  Errors as above plus INVALID_ARG for eps or NULL diff members. */
tdk_status tdk_diff_encode(tdk_round* r, int32_t layer, const tdk_layer_io* io, float eps,
                           const tdk_diff* out, void* hip_stream);

/* tdk_diff_encode for callers that cannot let the library own device allocations of its own choosing at
 * call time: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, same kernels and bit-identical results, but the per-(agent, page) flag bytes live in a static
 * device array inside the library (TDK_STATIC_SCRATCH_BYTES per GPU, held until the process ends) instead of
 * the round's allocation.  Calls no hipMalloc / hipFree and takes no timing events.  A round with more than
 * TDK_STATIC_SCRATCH_BYTES (agent, page) pairs is refused with TDK_ERR_CAPACITY before anything is enqueued.
 * All calls on one GPU share the array (the compare kernel rewrites every flag of its round, so earlier
 * contents never matter): calls that overlap in time on one GPU race, whatever their rounds or streams. */
#define TDK_STATIC_SCRATCH_BYTES (4u << 20)
tdk_status tdk_diff_encode_static(tdk_round* r, int32_t layer, const tdk_layer_io* io, float eps,
                                  const tdk_diff* out, void* hip_stream);

/* Writes every agent's shared span: pages listed in the diff from the payload, all others from the
 * re-rotated master.  `in` must hold what tdk_diff_encode produced for this round (ascending
 * indices); entries at or past capacity_pages are ignored (those pages come from the master). */
tdk_status tdk_diff_decode(tdk_round* r, int32_t layer, const tdk_layer_io* io, const tdk_diff* in,
                           void* hip_stream);

/* Single-plane diffs (Sec. 5: K and V keep separate block-index lists unless both touch the same
 * blocks; the single-plane kernel of "Fused Sparse Restore").  plane = TDK_PLANE_K or TDK_PLANE_V.
 * Same as tdk_diff_encode / tdk_diff_decode restricted to one plane: only that plane is compared,
 * listed, stored and restored; payload is [capacity_pages][T][H][D] (one plane per slot). */
#define TDK_PLANE_K 1
#define TDK_PLANE_V 2
tdk_status tdk_diff_encode_plane(tdk_round* r, int32_t layer, const tdk_layer_io* io, float eps, int32_t plane,
                                 const tdk_diff* out, void* hip_stream);
tdk_status tdk_diff_decode_plane(tdk_round* r, int32_t layer, const tdk_layer_io* io, int32_t plane,
                                 const tdk_diff* in, void* hip_stream);

/* Reuse plan of the check layer (Sec. 4.2 "Layerwise Collective Reuse" and "Reuse Plan Output"), all DEV,
 * caller-owned.
 *   score[sum_i S_i]              per-token deviation of agent i at master token m, agents in order:
 *                                 sum over the K row of (fresh - rotated cached)^2 in fp32, where fresh
 *                                 is the agent's K row in the pool and rotated cached is what
 *                                 tdk_rerotate_round would write there
 *   important[n_agents][k_stride] the agent's important positions (master token numbers), ascending
 *   n_important[n_agents]         how many there are: min(ceil(ratio * S), #tokens with !(score <= min_score))
 *   total[n_agents]               the agent's accumulated deviation (sum of its scores)
 *   master[n_sessions]            agent with the lowest total in each session (first one on ties, NaN
 *                                 totals count as +inf, -1 for a session without agents) */
typedef struct {
  float*   score;
  int32_t* important;
  int32_t  k_stride;      /* >= ceil(ratio * S) of every session that has agents */
  int32_t* n_important;
  float*   total;
  int32_t* master;
} tdk_reuse_plan;

/* One batched key-difference pass over the whole group on the check layer, selection of the
 * important positions of every request (the ceil(ratio * S) largest scores among tokens with
 * !(score <= min_score); ties go to the lower token number) and the choice of each session's master.
 * Reads pool_k and master_k only.  0 < ratio <= 1, min_score finite and >= 0. */
tdk_status tdk_check_layer(tdk_round* r, int32_t layer, const tdk_layer_io* io, float ratio, float min_score,
                           const tdk_reuse_plan* out, void* hip_stream);

/* Attention of new query tokens over the shared span of every mirror, from master + diff, with no
 * restored copy (Sec. 4.4, last paragraphs: applying the diff as attention tiles are loaded; Fig. 9:
 * identical blocks go straight to attention, blocks with a diff are corrected first).  All DEV.
 *   q          bf16 [n_agents][n_q][n_q_heads][D], rotated for the queries' own positions (all of them
 *              after the shared span: no causal mask inside it); n_q_heads a multiple of H, query head
 *              hq reads KV head hq / (n_q_heads / H)
 *   out        fp32 [n_agents][n_q][n_q_heads][D]: softmax(scale * q . K_i) V_i over the S tokens of the
 *              span, where (K_i, V_i) is the agent's mirror: payload rows on the pages its diff lists,
 *              the master's K rotated to the agent's offset and the master's V everywhere else
 *   lse        fp32 [n_agents][n_q][n_q_heads]: log of the softmax denominator, so that the caller can
 *              merge `out` with attention over the agent's private tokens (-inf, out 0 for an empty span)
 *   workspace  tdk_attend_workspace_bytes(r, n_q, n_q_heads) bytes, 256-byte aligned, contents undefined
 * Arithmetic: each query row is rotated back by the agent's offset (fp32, rounded to bf16) so that all
 * agents of a session multiply the same un-rotated master tiles (bf16 MFMA, fp32 accumulation, softmax
 * weights rounded to bf16 for the second product); the listed pages go through the same products
 * from the payload.  The result agrees with the exact definition to about 1e-2 of the largest |V| at
 * scale = 1 / sqrt(128), in proportion for larger scales (not bit for bit).  Any finite scale is taken:
 * the kernels work with its magnitude and the query copies carry its sign; zero (taken as 1e-30) gives uniform weights.
 * Scaled scores have to stay below 2^24 in magnitude: the reference point of a row is rounded after scaling. */
typedef struct {
  const void* q;
  int32_t     n_q;
  int32_t     n_q_heads;
  float       scale;
  float*      out;
  float*      lse;
  void*       workspace;
  size_t      workspace_bytes;
} tdk_attend_io;

size_t tdk_attend_workspace_bytes(const tdk_round* r, int32_t n_q, int32_t n_q_heads);   /* 0 on bad arguments */

/* io: master_k / master_v of the layer (the pool is not touched and may be NULL); in: the mirrors'
 * paired diff as tdk_diff_encode wrote it.  All layouts: identity or per-agent segments (one rotated copy
 * of a query row per segment), diffs stored at the current or at other positions (diff_pos0 / diff_pos).
 * Master values must be finite.
 * The workspace holds partial results.  tdk_attend_workspace_bytes never gets smaller with n_q: what it asks for n_q
 * query tokens serves every call on the round with fewer (a shorter call may be cut into more parts, and need more, than a
 * longer one).  A call with few query rows in the master's order that brings less is cut into fewer parts, as long as parts of 512
 * tokens or more fit: slower, and rounded at other places.  Other calls, and those with less, are refused.
 * Allocates nothing, enqueues one to four kernels, does not synchronise.  Errors: INVALID_ARG (NULL,
 * misaligned, n_q < 1, n_q_heads not a multiple of H, scale not finite, workspace too small). */
tdk_status tdk_attend_shared(tdk_round* r, int32_t layer, const tdk_layer_io* io, const tdk_diff* in,
                             const tdk_attend_io* a, void* hip_stream);

/* Round-aware prompt interface (Sec. 4.1) and segment-based index (Sec. 5), HOST only.  Prompts are
 * split at a reserved separator token; a block is identified by its content (64-bit hash index,
 * every hit confirmed by comparison), so a shared update is recognised at whatever position it sits.
 * A content held by at least two prompts is shared; prompts that hold the same set of shared contents
 * (at least two prompts) form a session, numbered by first prompt; the session's master lists the
 * shared blocks in the order of its first prompt (span = their total length); each member gets the
 * segment list tdk_agent takes (src_tok in that master, dst_pos = position in the member's prompt,
 * diff_pos = dst_pos).  Other prompts get session -1 (the single-request path).  Empty blocks are
 * ignored; of a content repeated inside one prompt the first occurrence counts.  Token arrays are
 * borrowed during the call only. */
typedef struct {
  const int32_t* tokens;   /* HOST */
  int32_t        n_tokens;
} tdk_prompt;
typedef struct tdk_prompt_plan tdk_prompt_plan;   /* opaque, host memory */
tdk_status tdk_prompt_plan_create(const tdk_prompt* prompts, int32_t n_prompts, int32_t separator,
                                  tdk_prompt_plan** out);   /* INVALID_ARG, NOMEM, UNSUPPORTED (span >= 2^31) */
void       tdk_prompt_plan_destroy(tdk_prompt_plan* p);     /* NULL-safe */
int32_t    tdk_prompt_plan_n_sessions(const tdk_prompt_plan* p);
int32_t    tdk_prompt_plan_span(const tdk_prompt_plan* p, int32_t session);         /* -1 if out of range */
int32_t    tdk_prompt_plan_session_of(const tdk_prompt_plan* p, int32_t prompt);    /* -1: none */
/* number of segments of a prompt (0 if it has no session, -1 if out of range); *out points into the
 * plan and stays valid until the plan is destroyed */
int32_t    tdk_prompt_plan_segments(const tdk_prompt_plan* p, int32_t prompt, const tdk_segment** out);

/* Ping-pong staging buffers of the layerwise restore, DEV, caller-owned: two K and two V buffers of
 * stage_bytes each, stage_bytes >= (sum_s S_s) * H * D * 2 (one layer of masters). */
typedef struct {
  void*  stage_k[2];
  void*  stage_v[2];
  size_t stage_bytes;
} tdk_pingpong;

/* Algorithm 1 (Sec. 4.4) for layers first_layer .. first_layer + n_layers - 1 of every mirror of the
 * round: the masters of layer k are copied from HOST memory (host_master_k[k], host_master_v[k];
 * pinned memory, layout as tdk_layer_io.master_k) into one staging buffer on copy_stream while the
 * previous layer, staged in the other buffer, is restored on compute_stream exactly as
 * tdk_diff_decode does (io[k].pool_*, diffs[k]; io[k].master_* are ignored).  Returns after
 * enqueueing; the result is complete when compute_stream has drained.  Uses events owned by the
 * round, so calls on one round must not be issued concurrently from several threads.  Errors: as
 * tdk_diff_decode for every layer (all checked before anything is enqueued), INVALID_ARG for NULL or
 * undersized staging. */
tdk_status tdk_restore_layers(tdk_round* r, int32_t first_layer, int32_t n_layers,
                              const void* const* host_master_k, const void* const* host_master_v,
                              const tdk_layer_io* io, const tdk_diff* diffs, const tdk_pingpong* pp,
                              void* compute_stream, void* copy_stream);

/* ---- The agents' own tokens -----------------------------------------------------------------------------
 * What a model does with the paged caches between two rounds: the tokens it has just computed are appended
 * (tdk_kv_append), their queries attend to the cache (tdk_kv_attend), and finished outputs leave it again as
 * the masters of the next round (tdk_kv_read).  One call covers a batch of sequences of any lengths; all of a
 * batch's description lies on the device, so a captured call serves every later step of the same sizes.
 *
 * A cache has one of three formats:
 *   TDK_KV_BF16    planes [pool_pages][T][H][D] bf16: the pool of the rounds (tdk_layer_io.pool_k / pool_v)
 *   TDK_KV_MXFP8   planes [pool_pages][H][T * 128 + T * 4] bytes, 1.94 times smaller: as MXFP4, but a value is a byte: one sign, four
 *                  exponent bits (bias 7) and three mantissa bits, magnitudes up to 448; 0x7f and 0xff are NaN.  A block's byte
 *                  255 makes all 32 NaN; values are infinite from 2^128 on (bytes from 247), and below 2^-124 (bytes 0 to 2, which append
 *                  does not write) they are rounded to bf16's grid of 2^-133.
 *   TDK_KV_MXFP4   planes [pool_pages][H][T * 64 + T * 4] bytes, 3.8 times smaller: per page and KV head the 4-bit
 *                  values of its T tokens (64 bytes each, element 2 i in the low half of byte i), then the
 *                  block exponents (4 bytes each).  A value is one sign, two exponent bits and one mantissa bit
 *                  (magnitudes 0 0.5 1 1.5 2 3 4 6); 32 consecutive elements of a row share a power of two
 *                  2^(byte - 127); byte 255 makes all 32 NaN.  Every call takes values as bf16 has them: exact, and
 *                  infinite from 2^128 on (bytes 253 and 254). */
#define TDK_KV_BF16  0
#define TDK_KV_MXFP4 1
#define TDK_KV_MXFP8 8

typedef struct tdk_kv tdk_kv;   /* opaque, host memory only: geometry, format, rotation frequencies, device */

/* num_layers of the model is not used.  A handle belongs to the device that is current when it is created; calls
 * with another device current fail with INVALID_ARG.  It holds no state between calls: calls may run at the
 * same time on several streams and from several threads.  Errors: INVALID_ARG, UNSUPPORTED (as
 * tdk_round_create; unknown format), NOMEM. */
tdk_status tdk_kv_create(const tdk_model* model, int32_t format, tdk_kv** out);
/* The same with positions that become angles by `rope`: tdk_kv_append and tdk_kv_rotate go by it. */
tdk_status tdk_kv_create_rope(const tdk_model* model, const tdk_rope* rope, int32_t format, tdk_kv** out);
void       tdk_kv_destroy(tdk_kv* kv);               /* NULL-safe; work that is enqueued already is not affected */
size_t     tdk_kv_page_bytes(const tdk_kv* kv);      /* bytes of one page in one plane; 0 for NULL */

/* One layer of a cache, DEV, 16-byte aligned. */
typedef struct {
  void*   k;
  void*   v;
  int64_t pool_pages;
} tdk_kv_cache;

/* A batch of sequences.  Sequence s has seq_len[s] tokens in all, and the last n_s = q_start[s + 1] - q_start[s]
 * of them are the batch's: its token t (position seq_len[s] - n_s + t) is row q_start[s] + t of the token buffers.
 *   n_tokens   rows of the token buffers; q_start[n_seqs] may be smaller: the rows behind it are left alone
 *   max_len    longest sequence that is expected: how a call is cut into workgroups goes by it and by the
 *              sizes above, and with that the order of its fp32 sums (a longer sequence is served too, only more slowly)
 * Token j lies in physical page block_table[s][j / T].  q_start must not decrease.  Everything on the device is
 * checked there: starts are cut to [0, n_tokens], and a token whose position is negative, whose logical page
 * lies past table_stride or whose page number is not in [0, pool_pages) is not written by append, reads as zero
 * and is seen by no query.  At most 2^30 sequences, 2^30 tokens per sequence by its table, and per call what one launch
 * holds: 2^32 threads, 256 for each token that is appended, read or rotated (else UNSUPPORTED). */
typedef struct {
  int32_t        n_seqs;
  int32_t        n_tokens;
  int32_t        max_len;
  const int32_t* q_start;       /* DEV [n_seqs + 1] */
  const int32_t* seq_len;       /* DEV [n_seqs]     */
  const int32_t* block_table;   /* DEV [n_seqs][table_stride] */
  int32_t        table_stride;
} tdk_kv_batch;

/* Rows of tokens, DEV, bf16, 16-byte aligned.  Row r of k starts at element r * k_stride and holds [H][D]; strides
 * are multiples of 8, at least H * D (n_q_heads * D), so that k, v and q may be slices of one projection's output. */
typedef struct {
  void*       k;
  void*       v;
  int64_t     k_stride;
  int64_t     v_stride;
  const void* q;                /* tdk_kv_append only: queries to rotate as well, or NULL */
  int64_t     q_stride;
  int32_t     n_q_heads;
  void*       q_out;            /* may be q itself, with the same stride */
  int64_t     q_out_stride;
} tdk_kv_rows;

/* Writes the batch's tokens into the cache: K (un-rotated in `rows`) rotated for each token's position in the
 * arithmetic above, V as it is; with q, the rotated queries into q_out.  MXFP4: the fp32 values go to the nearest
 * 4-bit value of their block (ties to even); the block's power of two is 2^(floor(log2 m) - 2) of its largest
 * magnitude m, one higher from m = 1.75 * 2^n on (what lies beyond 6 becomes 6), and 2^-126 at least; a block with an
 * infinity or NaN becomes NaN, and in one with m from 1.75 * 2^127 on what rounds to 2^128 is infinite.  MXFP8: the same with
 * 2^(floor(log2 m) - 8), one higher above 1.8125 * 2^n (what lies up to there becomes 448), and 2^-124 at least; in a block
 * with m above 1.8125 * 2^127 what rounds to 2^128 is infinite.  No two
 * tokens of a batch may have the same place in the cache (sequences that share pages differ in the pages they
 * append to).  One kernel. */
tdk_status tdk_kv_append(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch,
                         const tdk_kv_rows* rows, void* hip_stream);

/* Rows that are rotated and stay rows: the batch's keys on their way to tdk_prompt_attend, queries, or, with `back`, keys out of a cache
 * turned back to no position (the inverse: cosines and sines divided by the magnitude, the other way round).  Positions, starts and rows as in
 * tdk_kv_append; max_len, block_table and table_stride of the batch are not looked at, and rows of no sequence or with a negative position are left
 * alone.  Either plane may be NULL; out may be the source itself, with the same stride, and overlaps it nowhere else.  The handle's format does
 * not matter.  One kernel. */
typedef struct {
  const void* k;                /* rows [H][D] */
  int64_t     k_stride;
  void*       k_out;
  int64_t     k_out_stride;
  const void* q;                /* rows [n_q_heads][D] */
  int64_t     q_stride;
  int32_t     n_q_heads;
  void*       q_out;
  int64_t     q_out_stride;
  int32_t     back;
} tdk_kv_rotate_io;

tdk_status tdk_kv_rotate(const tdk_kv* kv, const tdk_kv_batch* batch, const tdk_kv_rotate_io* io, void* hip_stream);

/* The inverse: the batch's tokens out of the cache into rows->k / rows->v (the same rows that append would take;
 * K stays rotated; 4-bit values as above).  rows->q must be NULL.  One kernel. */
tdk_status tdk_kv_read(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch,
                       const tdk_kv_rows* rows, void* hip_stream);

/* Attention of the batch's tokens to their sequences.  The query at position p of sequence s sees token j iff
 *   j <= p,  and  window = 0 or j > p - window or j < n_sink,  and not hole[s][0] <= j < hole[s][1].
 *   q          bf16 rows [n_q_heads][D], rotated; query head hq reads KV head hq / (n_q_heads / H)
 *   out        bf16 rows [n_q_heads][D]: softmax(scale * q . K) V over what the query sees; zero if it sees nothing
 *   lse        fp32 [n_tokens][n_q_heads]: log of the softmax denominator, -inf for a query that sees nothing; may be NULL
 *   hole       DEV int32 [n_seqs][2], or NULL: tokens attended to elsewhere (the shared span, tdk_attend_shared)
 *   part_out, part_lse   DEV fp32 [n_tokens][n_q_heads][D] and [n_tokens][n_q_heads], or NULL: a partial result over other
 *              tokens, as tdk_attend_shared leaves it; out and lse are then those of both parts together
 *   workspace  tdk_kv_attend_workspace_bytes() bytes, 256-byte aligned, contents undefined; calls that may run at the same
 *              time (two streams, two graphs) need one each
 * Any scale up to 2^127 in magnitude is taken, zero and denormal ones as they are (scores q . K beyond fp32 are infinite
 * before they are scaled; a query all of whose scores are minus infinity counts as one that sees nothing).  What a query
 * does not see does not reach its result, whatever it holds (NaN and infinities included).  What it does see does: a NaN in V makes its element
 * NaN, an infinity makes it infinite, or NaN where it meets the other one or its weight is below fp32's range.  bf16 products with fp32 sums;
 * the softmax weights are rounded to bf16 for the second product, their sum is not.  Allocates nothing, one or two
 * kernels, does not synchronise; results do not depend on what else runs. */
typedef struct {
  const void*    q;
  int64_t        q_stride;      /* elements, a multiple of 8, at least n_q_heads * D */
  int32_t        n_q_heads;
  float          scale;
  void*          out;
  int64_t        out_stride;
  float*         lse;
  void*          workspace;
  size_t         workspace_bytes;
  int32_t        window;        /* 0: none */
  int32_t        n_sink;        /* first tokens that stay visible behind a window */
  const int32_t* hole;
  const float*   part_out;
  const float*   part_lse;
} tdk_kv_attend_io;

/* Depends on n_seqs, n_tokens and max_len only (nothing on the device is read); 0 where none is needed or on bad arguments. */
size_t     tdk_kv_attend_workspace_bytes(const tdk_kv* kv, const tdk_kv_batch* batch, int32_t n_q_heads);
tdk_status tdk_kv_attend(const tdk_kv* kv, const tdk_kv_cache* cache, const tdk_kv_batch* batch,
                         const tdk_kv_attend_io* a, void* hip_stream);

/* Attention of prompts that are not in pages: packed sequences, keys and values straight from the projections (rotated by
 * tdk_kv_rotate).  Sequence s has the keys k_start[s] .. k_start[s + 1] - 1 of the rows k and v, and the queries q_start[s] .. q_start[s + 1] - 1;
 * its queries are its last tokens: query t of n sees key j iff j <= p = n_keys - n + t, and window = 0 or j > p - window or j < n_sink.  Queries of
 * a sequence with fewer keys than queries that come before the first key see nothing.  A prompt's first pass has as many queries as
 * keys (both arrays may be one); a later chunk has all keys so far.  Starts must not decrease and are cut to [0, n_q] and [0, n_k];
 * queries of no sequence are left alone.
 *   n_q, n_k     rows of q and out, rows of k and v
 *   max_len      keys of the longest sequence that is expected, as in tdk_kv_batch
 * The handle gives the heads and the device; its format and frequencies do not matter. */
typedef struct {
  int32_t        n_seqs;
  int32_t        n_q;
  int32_t        n_k;
  int32_t        max_len;
  const int32_t* q_start;       /* DEV [n_seqs + 1] */
  const int32_t* k_start;       /* DEV [n_seqs + 1] */
} tdk_prompt_batch;

/* As tdk_kv_attend_io, with rows k and v of [H][D] bf16 (strides at most 2^24 elements).  out_f32: out is fp32 (out_stride in elements of
 * it), so that it can be another call's part_out: a prompt attends to its own rows here and to its history in the pages with
 * tdk_kv_attend, whose hole is the prompt's span.  It saves the rounding of the result, not that of the weights to bf16, which is in it as in every
 * result of these calls: 2^-8 of the weighted sum of |V| at most. */
typedef struct {
  const void*    q;
  int64_t        q_stride;
  int32_t        n_q_heads;
  const void*    k;
  int64_t        k_stride;
  const void*    v;
  int64_t        v_stride;
  float          scale;
  void*          out;
  int64_t        out_stride;
  int32_t        out_f32;
  float*         lse;
  void*          workspace;
  size_t         workspace_bytes;
  int32_t        window;
  int32_t        n_sink;
  const float*   part_out;
  const float*   part_lse;
} tdk_prompt_attend_io;

/* Depends on n_seqs, n_q, n_k and max_len only; 0 where none is needed or on bad arguments. */
size_t     tdk_prompt_attend_workspace_bytes(const tdk_kv* kv, const tdk_prompt_batch* batch, int32_t n_q_heads);
tdk_status tdk_prompt_attend(const tdk_kv* kv, const tdk_prompt_batch* batch, const tdk_prompt_attend_io* io, void* hip_stream);

/* Storage arithmetic of Sec. 6.4 (host only). */
double tdk_dense_bytes(const tdk_model* m, int64_t span_tokens);   /* one layer of one cache      */
double tdk_diff_bytes(const tdk_model* m, int64_t diff_pages);     /* values + idx + count/offset */
double tdk_family_cost(int64_t n_agents, double ratio);            /* 1 + (N-1)/R full caches     */

#ifdef __cplusplus
}
#endif
#endif
