// Launch descriptor of the differential attention calls, shared by the host
// dispatcher (kvt_api.cpp) and kvt_diff*.hip; travels by value.
#pragma once

#include "kvt_internal.h"

namespace kvt {

// Differential attention tiling: one workgroup = 8 waves, two maps x 4 blocks of 32 packed query rows.
constexpr int kDiffWaves = 8;
constexpr int kDiffTileRows = kDiffWaves / 2 * 32;
constexpr int kDiffDecHeads = 16;   // decode: query heads per workgroup, two maps each on one 32-row block

// Differential attention: extend and decode units, and the join of key splits
// (there the sequences that are split, unit_begin counting their rows).
struct DiffArgs {
  const void* q;
  const void* k_pool;
  const void* v_pool;
  void* out;
  const float* lambda;        // + token * lambda_stride + head
  const float* norm_weight;   // [D], or null: no norm
  float* part_o;              // [partial row][2][D]: unnormalised outputs of both maps
  float* part_ml;             // [partial row][4]: (running max in log2 units, row sum) of both maps
  const int32_t* block_table;
  int64_t lambda_stride;
  int64_t num_blocks;
  int32_t max_blocks;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t group;              // Hq / Hkv
  float scale_log2;           // scale * log2(e)
  float eps;
  float out_scale;
  int32_t nseq;
  uint8_t nsplit[kSeqsPerLaunch];          // key splits of each sequence; 1: its units write out themselves
  uint8_t nlast[kSeqsPerLaunch];           // extend: key splits of its last row tile (at most nsplit)
  int32_t part_row[kSeqsPerLaunch];        // first partial row of a split sequence: [split][token][head]
  int32_t unit_begin[kSeqsPerLaunch + 1];  // prefix sums of the sequences' units
  SeqDesc seq[kSeqsPerLaunch];
};
static_assert(sizeof(DiffArgs) <= 8192, "kernel argument block too large");

hipError_t launch_diff_extend(const DiffArgs& a, int dtype, int head_dim, int grid, hipStream_t stream);
hipError_t launch_diff_decode(const DiffArgs& a, int dtype, int head_dim, int grid, bool one_per_cu, hipStream_t stream);
hipError_t launch_diff_combine(const DiffArgs& a, int dtype, int head_dim, hipStream_t stream);

}  // namespace kvt
