// Caches that programs append to (tdk_kv_*): what the host side hands to the kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tdk.h"
#include "tdk_types.h"

namespace tdk {

// A batch and the cache it goes to.
struct KvDev {
  char*          k;
  char*          v;
  int32_t        pool_pages;
  const int32_t* q_start;
  const int32_t* seq_len;
  const int32_t* table;
  int32_t        table_stride;
  int32_t        n_seqs;
  int32_t        n_tokens;
  int32_t        heads;        // H
  int32_t        page_shift;   // log2 T
  int32_t        interleaved;
};

// The formats of pages.
constexpr int kBf16 = 0, kMx4 = 4, kMx8 = 8;

// Rows in and out of the cache.
struct KvRowsDev {
  char*       k;
  char*       v;
  const char* q;
  char*       q_out;
  int64_t     k_stride, v_stride, q_stride, q_out_stride;   // bytes
  int32_t     n_q_heads;       // 0: no queries
  int32_t     waves;           // workgroups per token
  double      inv_freq[kHalf];                              // of the pairs that turn, zero behind them
  int32_t     rotary;          // elements of a head that turn
  double      magnitude;       // of their cosines and sines
};

// Rows that are only rotated.
struct KvRotateDev {
  const char* k;               // NULL: none
  const char* q;
  char*       k_out;
  char*       q_out;
  int64_t     k_stride, k_out_stride, q_stride, q_out_stride;   // bytes
  int32_t     n_k_heads, n_q_heads;                         // 0: none
  int32_t     waves;           // wavefronts per token: in one workgroup (many tokens) or in as many
  int32_t     rotary;
  double      cos_size, sin_size;                           // factors of the cosines and sines
  double      inv_freq[kHalf];
};

// Attention.
struct KvAttendDev {
  const char*    q;
  char*          out;
  float*         lse;
  float*         part_o;       // workspace: [n_tokens * n_q_heads][n_chunks][128] un-normalised partial outputs
  float*         part_ml;      // workspace: [n_tokens * n_q_heads][n_chunks][2] reference point (a score), sum
  const int32_t* hole;
  const float*   other_out;    // the caller's partial result
  const float*   other_lse;
  int64_t        q_stride, out_stride;                      // bytes
  int32_t        n_q_heads;
  int32_t        group;        // query heads per KV head
  int32_t        window, n_sink;
  int32_t        n_chunks;     // parts of a sequence at most, each a workgroup's
  int32_t        piece_tiles;  // tiles of a part
  int32_t        n_rest;       // row blocks times parts
  int32_t        q_flip;       // the caller's scale was negative: the queries carry the sign
  float          scale;        // its magnitude, not zero
  float          scale2;       // times log2(e)
  uint32_t       group_inv;    // 2^22 / group, rounded up
  int32_t        last_id;      // row blocks from this number down; -1: from 0 up
};

// Attention of rows that are not in pages: KvDev has the rows (k, v, q_start; no table), the base what both kinds share.
struct PromptAttendDev : KvAttendDev {
  const int32_t* k_start;
  int64_t        k_stride, v_stride;                        // bytes
  int32_t        n_k;          // rows of k and v
  int32_t        f32;          // out is fp32
  int32_t        down;         // row blocks: so many from last_id down, the others from 0 up
};

// How a call of the attention is cut.
struct KvAttendPlan {
  int32_t block_rows = 16;     // query rows (token, head of the group) per workgroup
  bool forward = true;         // one block per sequence on average: the blocks in their order (else backward)
  int64_t ids = 0;             // row blocks: an upper bound over all ways the tokens can be spread over the sequences
  int32_t n_chunks = 1;
  int32_t piece_tiles = 1;
  int64_t rows = 0;            // n_tokens * n_q_heads
  size_t  o_part_ml = 0, bytes = 0;
};

// many: a call whose rows the caches would not hold for whoever comes next
hipError_t launch_kv_append(const KvDev& kv, const KvRowsDev& rows, int fmt, bool many, hipStream_t st);
hipError_t launch_kv_append_rope(const KvDev& kv, const KvRowsDev& rows, int fmt, bool many, hipStream_t st);
hipError_t launch_kv_rotate(const KvDev& kv, const KvRotateDev& r, bool many, hipStream_t st);
hipError_t launch_kv_read(const KvDev& kv, const KvRowsDev& rows, int fmt, bool many, hipStream_t st);
hipError_t launch_kv8_read(const KvDev& kv, const KvRowsDev& rows, bool many, hipStream_t st);
hipError_t launch_kv_attend(const KvDev& kv, const KvAttendDev& at, const KvAttendPlan& p, int fmt, hipStream_t st);
hipError_t launch_kv8_attend(const KvDev& kv, const KvAttendDev& at, const KvAttendPlan& p, int64_t blocks, hipStream_t st);
hipError_t launch_prompt_attend(const KvDev& kv, const PromptAttendDev& at, const KvAttendPlan& p, hipStream_t st);
hipError_t launch_kv_join(const KvDev& kv, const KvAttendDev& at, int64_t rows, hipStream_t st);

}  // namespace tdk
