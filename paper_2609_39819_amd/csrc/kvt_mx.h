// Launch descriptors of the calls over 4-bit pages and of eviction
// (kvt_mx_append.hip, kvt_mx_extend.hip, kvt_mx_decode.hip, kvt_weights.hip,
// kvt_evict.hip); the extend call over 4-bit pages takes ExtendArgs.
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

// Attention of few query rows (a decoding step, a short chunk).  The tiles of
// kDecKeysPerTile keys of a launch's sequences lie one after the other, and slot x
// of a kv-head takes tiles x * share .. (x + 1) * share - 1: parts of as many
// sequences as lie there.  share 0: slot x is sequence x.  A sequence in more than
// one slot leaves a partial result in each, parts of them from row part_row on,
// [parts][S_b * Hq].
struct MxDecodeArgs {
  const void* q;
  const void* k_pool;
  const void* v_pool;
  void* out;
  float* lse;           // may be null
  float* part_o;        // [partial rows][D]
  float* part_ml;       // [partial rows][2]  (reference max in log2 units, row sum)
  const int32_t* block_table;
  int64_t num_blocks;
  int32_t max_blocks;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;        // Hq / Hkv
  int32_t chunks;       // workgroups that share the rows of a kv-head (S_b * group), of the launch's largest
  float scale_log2;
  int32_t share;
  int32_t nseq;
  int32_t tile_begin[kSeqsPerLaunch + 1];
  int32_t part_row[kSeqsPerLaunch];
  SeqDesc seq[kSeqsPerLaunch];
};
constexpr int kMxChunkRows = 32;   // rows of a workgroup at most
constexpr int kMxMaxParts = 255;   // slots that hold a part of one sequence at most
// Rows of a kv-head up to which an extend call counts as one of few.  32/8 heads of
// 128, by the chunks of the decode kernel and by the extend kernel: 64 rows over 4000
// keys 17.9 and 17.7 us, over 131000 67.6 and 97.8; 128 rows 19.6 and 23.1, 112.7
// and 101.3, over 32000 42.9 and 37.3.
constexpr int kMxFewRows = 64;

// The join of a launch's split sequences.
struct MxJoinArgs {
  const float* part_o;
  const float* part_ml;
  void* out;
  float* lse;
  int32_t nseq;
  int32_t row_begin[kSeqsPerLaunch + 1];   // prefix sums of the sequences' rows (S_b * Hq)
  int32_t part_row[kSeqsPerLaunch];
  int32_t row[kSeqsPerLaunch];             // first output row
  uint8_t parts[kSeqsPerLaunch];
};

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
  uint32_t by_group;    // x / group = (x * by_group >> 32) >> group_shift for x < 2 * group + 256, group > 1
  int32_t group_shift;
  float scale_log2;
  int32_t share;        // step kernel: tiles of a workgroup
  int32_t tiles;        // turn kernel: of a workgroup, if every sequence's rows are one stage; else 0
  int32_t nseq;
  int32_t unit_begin[kSeqsPerLaunch + 1];   // prefix sums of the sequences' tiles (step kernel) or wide workgroups
  int32_t narrow_begin[kSeqsPerLaunch + 1]; // turn kernel: of the narrow ones, for the keys after those
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
  int32_t first_block;      // move kernel: of this launch
  int32_t unit_begin[kSeqsPerLaunch + 1];   // move kernel: prefix sums of the sequences' target pages
  EvictDesc seq[kSeqsPerLaunch];
};

static_assert(sizeof(MxRowsArgs) <= 8192 && sizeof(MxDecodeArgs) <= 8192 && sizeof(MxJoinArgs) <= 8192 && sizeof(WeightsArgs) <= 8192 && sizeof(EvictArgs) <= 8192,
              "kernel argument block too large");

hipError_t launch_mx_append(const MxRowsArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_mx_read(const MxRowsArgs& a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_mx_extend(const ExtendArgs& a, int dtype, int head_dim, int grid, hipStream_t stream);
hipError_t launch_mx_decode(const MxDecodeArgs& a, int dtype, int head_dim, int grid, hipStream_t stream);
hipError_t launch_mx_join(const MxJoinArgs& a, int dtype, int head_dim, hipStream_t stream);
// format: a kvt_dtype of the K pool, kMx for 4-bit pages, or kRounded for fp32
// pages and queries that are rounded to bf16 as the other attention calls round
// them (attention weights only); dtype is q's.
constexpr int kMx = 2;
constexpr int kRounded = 3;
hipError_t launch_weights_step(const WeightsArgs& a, int format, int dtype, int head_dim, int grid, hipStream_t stream);
hipError_t launch_weights_turn(const WeightsArgs& a, int format, int dtype, int head_dim, int grid, hipStream_t stream);
constexpr int kWeightsStepKeys = 32;      // step kernel: keys of one tile
constexpr int kWeightsWideKeys = 256;     // turn kernel: keys of a wide workgroup's tile (a narrow one's: 32)
constexpr int weights_stage_rows(int dtype) { return dtype == 0 ? 256 : 64; }   // turn kernel: rows in LDS at a time
hipError_t launch_evict_select(const EvictArgs& a, hipStream_t stream);
hipError_t launch_evict_move(const EvictArgs& a, int format, int head_dim, int blocks, hipStream_t stream);

}  // namespace kvt
