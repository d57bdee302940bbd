// Launch descriptor of the rotary calls, shared by the host dispatcher
// (kvt_api.cpp) and kvt_rotary.hip; travels by value.
#pragma once

#include "kvt_internal.h"

namespace kvt {

// Rotary positions of q rows, and of K rows on their way into the pages (with
// num_kv_heads = 0: q rows only, no sequences).  Strides in elements.
struct RotaryArgs {
  const void* q;       // null: no q rows (num_q_heads = 0)
  void* q_out;
  const void* k_new;
  const void* v_new;
  void* k_pool;
  void* v_pool;
  int64_t q_stride, q_out_stride, k_stride, v_stride;
  const int32_t* block_table;
  const int32_t* positions;   // [num_axes][total_rows], or null: the logical positions
  int64_t num_blocks;
  int64_t row_begin;          // first packed row covered by this launch
  int64_t rows;               // rows covered by this launch
  int64_t total_rows;         // T of the whole call
  int32_t max_blocks;
  int32_t num_q_heads, num_kv_heads;
  int32_t rot_dim;            // rotated columns of each part
  int32_t parts;
  int32_t interleaved;
  int32_t nseq;
  int32_t head_lanes;         // set by the launch: heads that a workgroup holds at a time
  uint8_t axis[64];           // axis of each frequency
  double turns[64];           // turns per position of each frequency
  SeqDesc seq[kSeqsPerLaunch];  // in packed-row order
};

static_assert(sizeof(RotaryArgs) <= 8192, "kernel argument block too large");

hipError_t launch_rotary(RotaryArgs& a, int dtype, int head_dim, int cus, hipStream_t stream);

}  // namespace kvt
