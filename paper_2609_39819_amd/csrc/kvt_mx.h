// Launch descriptors of the calls over 4-bit pages and of eviction
// (kvt_mx_append.hip, kvt_mx_extend.hip, kvt_mx_decode.hip, kvt_weights.hip,
// kvt_evict.hip); the attention calls over 4-bit pages take ExtendArgs.
#pragma once

#include "kvt_internal.h"

namespace kvt {

// A 4-bit page of one kv-head: the codes of 16 tokens, [16][D/2] bytes, then
// their scales, [16][D/32] bytes.
constexpr int mx_code_bytes(int head_dim) { return kBlock * head_dim / 2; }
constexpr int mx_page_bytes(int head_dim) { return kBlock * head_dim / 2 + kBlock * head_dim / 32; }

// New tokens' rows into 4-bit pages, or the values of such rows back.
struct MxRowsArgs {
  void* k;           // token rows, of dtype; read by append, written by read
  void* v;
  int64_t k_stride;  // elements from token to token
  int64_t v_stride;
  void* k_pool;      // 4-bit pages
  void* v_pool;
  const int32_t* block_table;
  int64_t num_blocks;
  int32_t max_blocks;
  int32_t num_kv_heads;
  int32_t row_begin;  // first packed row covered by this launch
  int32_t rows;       // rows covered by this launch
  int32_t nseq;
  SeqDesc seq[kSeqsPerLaunch];  // in packed-row order
};

// Query heads of one kv-head that one decode4 workgroup serves.
constexpr int kMxDecMaxRows = 32;

// Attention weights per position.
struct WeightsArgs {
  const void* q;
  const void* k_pool;
  const float* lse;
  float* weights;       // [B][Hkv][stride]
  int64_t stride;
  const int32_t* block_table;
  int64_t num_blocks;
  int32_t max_blocks;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;        // Hq / Hkv
  float scale_log2;
  int32_t nsplit;       // step kernel: workgroups per (sequence, kv-head)
  int32_t nseq;
  int32_t unit_begin[kSeqsPerLaunch + 1];
  SeqDesc seq[kSeqsPerLaunch];
};

struct EvictDesc {
  int32_t seq;
  int32_t length;   // L_b
  int32_t keep;     // n_b = min(L_b, keep_b)
};

struct EvictArgs {
  void* k_pool;
  void* v_pool;
  const float* weights;   // [B][Hkv][stride]
  int64_t stride;
  int32_t* positions;     // [B][Hkv][out_stride]
  float* weights_out;     // may be null
  int64_t out_stride;
  const int32_t* block_table;
  const int32_t* to_table;
  int64_t num_blocks;
  int32_t max_blocks;
  int32_t to_max_blocks;
  int32_t num_kv_heads;
  int32_t sinks;
  int32_t recent;
  int32_t nseq;
  int32_t unit_begin[kSeqsPerLaunch + 1];   // move kernel: prefix sums of the sequences' target pages
  EvictDesc seq[kSeqsPerLaunch];
};

static_assert(sizeof(MxRowsArgs) <= 8192 && sizeof(WeightsArgs) <= 8192 && sizeof(EvictArgs) <= 8192,
              "kernel argument block too large");

hipError_t launch_mx_append(const MxRowsArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_mx_read(const MxRowsArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_mx_extend(const ExtendArgs& a, int dtype, int head_dim, int grid, hipStream_t stream);
// chunks: workgroups that share a kv-head's query heads.  Every sequence has
// its own split count (ExtendArgs::last); nsplit is the number of partial sets.
hipError_t launch_mx_decode(const ExtendArgs& a, int dtype, int head_dim, int chunks, int grid, hipStream_t stream);
// format: a kvt_dtype of the K pool, or kMx for 4-bit pages; dtype is q's.
constexpr int kMx = 2;
hipError_t launch_weights_step(const WeightsArgs& a, int format, int dtype, int head_dim, int grid, hipStream_t stream);
hipError_t launch_weights_turn(const WeightsArgs& a, int format, int dtype, int head_dim, int waves, int grid,
                               hipStream_t stream);
int weights_keys_per_unit(int format);   // turn kernel: keys of one workgroup
hipError_t launch_evict_select(const EvictArgs& a, hipStream_t stream);
hipError_t launch_evict_move(const EvictArgs& a, int format, int head_dim, int grid, hipStream_t stream);

}  // namespace kvt
