// C-ABI entry points: argument validation, work planning and launches.
//
// Every check runs on the host before the first HIP call, so a bad call
// returns an error with nothing enqueued.  Planning is host arithmetic only:
// sequences are ordered longest first, the (row tile, key split) units of
// each sequence are numbered longest first, and the kv-head index varies
// fastest over workgroup ids -- workgroups are dispatched round-robin over the
// 8 XCDs, so with 8 (or a multiple/divisor of 8) kv-heads every workgroup of
// one kv-head runs on the same XCD and its K/V stream is shared in that L2.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>
#include <numeric>
#include <unordered_set>
#include <vector>

#include "kvt.h"
#include "kvt_diff.h"
#include "kvt_mx.h"
#include "kvt_internal.h"
#include "kvt_rotary.h"

namespace {

thread_local int g_last_hip_error = 0;

kvt_status device_error(hipError_t e) {
  g_last_hip_error = (int)e;
  return KVT_ERR_DEVICE;
}

int elem_bytes(int32_t dtype) { return dtype == KVT_DTYPE_BF16 ? 2 : 4; }

// Number of compute units of the current device, queried once per device
// (concurrent first calls may both query; they store the same value).
int device_cus() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) { (void)hipGetLastError(); return 256; }
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
      (void)hipGetLastError();
      n = 256;
    }
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// The kernels move 16-byte pieces of every token row, page and workspace.
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

kvt_status check_pool(const kvt_pool* pool) {
  if (pool == nullptr || pool->k == nullptr || pool->v == nullptr) return KVT_ERR_INVALID_ARG;
  if (!aligned16(pool->k) || !aligned16(pool->v)) return KVT_ERR_INVALID_ARG;
  if (pool->num_blocks < 1 || pool->num_kv_heads < 1) return KVT_ERR_INVALID_ARG;
  if (pool->head_dim != 64 && pool->head_dim != 128) return KVT_ERR_UNSUPPORTED;
  if (pool->dtype != KVT_DTYPE_BF16 && pool->dtype != KVT_DTYPE_F32) return KVT_ERR_UNSUPPORTED;
  return KVT_OK;
}

// Validates lengths and table width; fills the total token count.
kvt_status check_seqs(const kvt_seqs* seqs, int64_t* total_tokens) {
  if (seqs == nullptr || seqs->num_seqs < 1) return KVT_ERR_INVALID_ARG;
  if (seqs->prefix_len == nullptr || seqs->suffix_len == nullptr || seqs->block_table == nullptr)
    return KVT_ERR_INVALID_ARG;
  if (seqs->max_blocks < 1) return KVT_ERR_INVALID_ARG;
  int64_t T = 0;
  for (int b = 0; b < seqs->num_seqs; ++b) {
    const int64_t P = seqs->prefix_len[b], S = seqs->suffix_len[b];
    if (P < 0 || S < 1) return KVT_ERR_INVALID_ARG;
    const int64_t L = P + S;
    if (L > INT32_MAX / 2) return KVT_ERR_INVALID_ARG;
    if ((L + kvt::kBlock - 1) / kvt::kBlock > seqs->max_blocks) return KVT_ERR_INVALID_ARG;
    T += S;
  }
  if (T > INT32_MAX / 2) return KVT_ERR_INVALID_ARG;
  *total_tokens = T;
  return KVT_OK;
}

// Query heads: a positive multiple of the kv-heads, and T * num_q_heads
// packed query rows must fit the kernels' 32-bit row indices.
bool heads_ok(const kvt_pool* pool, int32_t num_q_heads, int64_t T) {
  if (num_q_heads < 1 || num_q_heads % pool->num_kv_heads != 0) return false;
  return T * num_q_heads <= INT32_MAX;
}

// Checked mode: every used block id is inside the pool.
kvt_status check_table_ids(const kvt_pool* pool, const kvt_seqs* seqs) {
  if (seqs->block_table_host == nullptr) return KVT_OK;
  for (int b = 0; b < seqs->num_seqs; ++b) {
    const int64_t L = (int64_t)seqs->prefix_len[b] + seqs->suffix_len[b];
    const int64_t nblk = (L + kvt::kBlock - 1) / kvt::kBlock;
    const int32_t* row = seqs->block_table_host + (int64_t)b * seqs->max_blocks;
    for (int64_t i = 0; i < nblk; ++i)
      if (row[i] < 0 || (int64_t)row[i] >= pool->num_blocks) return KVT_ERR_OUT_OF_RANGE;
  }
  return KVT_OK;
}

// Checked mode: two of the T new tokens may not target one (block, slot).  The set
// is made for all of them at once (grown step by step the search takes 4 % longer).
kvt_status check_append_targets(const kvt_seqs* seqs, int64_t T) {
  if (seqs->block_table_host == nullptr) return KVT_OK;
  std::unordered_set<int64_t> seen;
  seen.reserve((size_t)T * 2);
  for (int b = 0; b < seqs->num_seqs; ++b) {
    const int32_t* row = seqs->block_table_host + (int64_t)b * seqs->max_blocks;
    for (int32_t t = 0; t < seqs->suffix_len[b]; ++t) {
      const int64_t pos = (int64_t)seqs->prefix_len[b] + t;
      const int64_t key = (int64_t)row[pos / kvt::kBlock] * kvt::kBlock + pos % kvt::kBlock;
      if (!seen.insert(key).second) return KVT_ERR_OUT_OF_RANGE;
    }
  }
  return KVT_OK;
}

// Bytes of one kv-head's page, and of one of a pool's two tensors; `mx`: 4-bit pages.
int64_t page_bytes_of_head(const kvt_pool* pool, bool mx) {
  return mx ? kvt::mx_page_bytes(pool->head_dim) : (int64_t)kvt::kBlock * pool->head_dim * elem_bytes(pool->dtype);
}
size_t pool_tensor_bytes(const kvt_pool* pool, bool mx) {
  return (size_t)pool->num_blocks * pool->num_kv_heads * (size_t)page_bytes_of_head(pool, mx);
}

bool overlaps(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + bn && y < x + an;
}

// Workspace of nsplit partial results per packed row: the unnormalised
// outputs in fp32 (256-byte aligned block), then (m, l) in fp32.
size_t part_o_bytes(const kvt_pool* pool, int nsplit, int64_t rows) {
  return (((size_t)nsplit * rows * pool->head_dim * sizeof(float) + 255) / 256) * 256;
}
size_t part_bytes(const kvt_pool* pool, int nsplit, int64_t rows) {
  return part_o_bytes(pool, nsplit, rows) + (size_t)nsplit * rows * 2 * sizeof(float);
}

struct ExtendPlan {
  int nsplit = 1;
  int nsplit_base = 1;      // splits to fall back to when the workspace offered is too small for nsplit
  int nsplit_shared = 0;    // cascade only: key splits of the shared part
  bool use_shared = true;   // cascade only: false = run the plain extend plan
  double heaviest = 0.0;    // extend only: weight of the heaviest row tile when lighter ones take fewer splits, else 0
  std::vector<int> order;   // sequences, longest key range first
  size_t ws_bytes = 0;      // workspace needed for nsplit > 1
};

int row_tiles(int32_t suffix, int group) {
  const int64_t rows = (int64_t)suffix * group;
  return (int)((rows + kvt::kExtTileRows - 1) / kvt::kExtTileRows);
}

// Cost of the combine launch that merges split partials, in us.
constexpr double kMergeLaunchUs = 4.0;
// Fixed cost of one workgroup, in key tiles: its prologue (kernel arguments,
// block-table entries and the first tile's gather, about 3.3 us) and its
// epilogue.
constexpr double kUnitTiles = 2.0;

// CUs by the time they become free, as runs of equal times in ascending
// order, so that equal units on equally free CUs are placed in one step.  (A
// heap of the CUs is filled and popped unit by unit: it was most of the time
// of a cascade's plan.)
class FreeTimes {
 public:
  FreeTimes(double early, int64_t n_early, double late, int64_t n_late) {
    if (n_early > 0) runs_.push_back({early, n_early});
    if (n_late > 0) runs_.push_back({late, n_late});
  }
  // Puts `jobs` units of length len, one after the other, each on the CU that
  // is free first; returns the latest finish.
  double run(int64_t jobs, double len) {
    double last = 0;
    while (jobs > 0) {
      Run& first = runs_[head_];
      const int64_t n = std::min(jobs, first.count);
      const double t = first.time + len;
      jobs -= n;
      if ((first.count -= n) == 0) ++head_;
      auto at = std::lower_bound(runs_.begin() + head_, runs_.end(), t, [](const Run& r, double x) { return r.time < x; });
      if (at != runs_.end() && at->time == t) at->count += n;
      else runs_.insert(at, Run{t, n});
      last = t;   // the earliest free CU never gets earlier
    }
    return last;
  }
  // Time in which the CUs get through what they were given, if one of them works
  // at rate `one` at most and all of them share rate `all`.
  double drain(double one, double all) const {
    double t = 0, at = 0;
    int64_t left = 0;
    for (size_t i = head_; i < runs_.size(); ++i) left += runs_[i].count;
    for (size_t i = head_; i < runs_.size(); ++i) {
      t += (runs_[i].time - at) * std::max(1.0 / one, (double)left / all);
      at = runs_[i].time;
      left -= runs_[i].count;
    }
    return t;
  }

 private:
  struct Run {
    double time;
    int64_t count;
  };
  std::vector<Run> runs_;
  size_t head_ = 0;
};

// Finish time, in key tiles, of one extend launch: list scheduling of its
// units in launch order onto the CUs (each unit to the CU that frees first,
// as workgroups are dispatched): shared_jobs units of len_s tiles first
// (a cascade's shared part; none for a plain extend), then each sequence's
// units (jobs_p[b] row tiles of ceil(kt_p[b] / ns_p) tiles, ns_p splits
// each, of which one in `share` falls to the CUs modelled); every unit also
// pays kUnitTiles.  Callers model one kv-head's units on its share of the
// CUs (the units of the kv-heads alternate) or one XCD's (workgroups go to
// the XCDs in turn).
double list_finish(int64_t shared_jobs, double len_s, const std::vector<int64_t>& jobs_p,
                   const std::vector<int64_t>& kt_p, int ns_p, int cus, int share = 1) {
  const int64_t rounds = shared_jobs / cus, rest = shared_jobs % cus;
  const double early = (double)rounds * (len_s + kUnitTiles), late = (double)(rounds + 1) * (len_s + kUnitTiles);
  FreeTimes free_at(early, cus - rest, late, rest);
  double span = rest > 0 ? late : early;
  for (size_t b = 0; b < jobs_p.size(); ++b) {
    const double len = std::ceil((double)kt_p[b] / ns_p) + kUnitTiles;
    span = std::max(span, free_at.run((jobs_p[b] * ns_p + share - 1) / share, len));
  }
  return span;
}

// Sequences in launch order, longest key range first (stable).
std::vector<int> longest_first(const kvt_seqs* seqs) {
  std::vector<int> order(seqs->num_seqs);
  std::iota(order.begin(), order.end(), 0);
  if (order.size() > 1)
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) {
      return (int64_t)seqs->prefix_len[x] + seqs->suffix_len[x] > (int64_t)seqs->prefix_len[y] + seqs->suffix_len[y];
    });
  return order;
}

// Split long key ranges only when the row tiles alone cannot fill the chip.
ExtendPlan make_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads, int64_t T, int cus) {
  ExtendPlan p;
  const int B = seqs->num_seqs;
  const int G = num_q_heads / pool->num_kv_heads;
  p.order = longest_first(seqs);
  int64_t units = 0;
  int64_t min_keys = INT64_MAX, min_len = INT64_MAX, max_len = 0;
  for (int b = 0; b < B; ++b) {
    units += (int64_t)row_tiles(seqs->suffix_len[b], G) * pool->num_kv_heads;
    min_keys = std::min<int64_t>(min_keys, (int64_t)seqs->prefix_len[b] + 1);
    const int64_t len = (int64_t)seqs->prefix_len[b] + seqs->suffix_len[b];
    min_len = std::min(min_len, len);
    max_len = std::max(max_len, len);
  }
  // Split the key range when whole rounds of workgroups over the CUs leave
  // many CUs idle: with ns splits a unit's work shrinks to 1/ns and the call
  // takes about ceil(units*ns / cus) / ns unit-times.  Take the smallest ns
  // with the best estimate if it beats no split by at least 10 %; each split
  // keeps at least 16 key tiles (1024 keys) of the shortest sequence.
  const int64_t by_keys = std::max<int64_t>(1, min_keys / (16 * kvt::kExtKeysPerTile));
  const int ns_max = (int)std::min<int64_t>(by_keys, kvt::kMaxSplits);
  auto rounds = [&](int s) { return (double)((units * s + cus - 1) / cus) / s; };
  int ns = 1;
  for (int s = 2; s <= ns_max; ++s)
    if (rounds(s) < rounds(ns) - 1e-9) ns = s;
  if (rounds(ns) > 0.9 * rounds(1)) ns = 1;
  // Ragged batches: the rule above counts units as equal and keeps 1024 keys
  // of the shortest sequence per split, so one short sequence stops the long
  // ones from splitting.  When the longest key range is more than twice the
  // shortest and the row tiles fit a few rounds of the CUs, list-schedule
  // the launch for 1, 2, 4, 8 and 16 splits (one XCD's eighth of the units
  // on its CUs, each unit's length from its sequence's key tiles) and take
  // the best finish plus partial cost if it beats the rule's choice by more
  // than a fifth.
  constexpr int kXcds = 8;
  const int xcd_cus = std::max(1, cus / kXcds);
  if (max_len > 2 * min_len && units <= 4 * (int64_t)cus) {
    const int64_t rows = T * num_q_heads;
    std::vector<int64_t> jobs(B), kt(B);
    for (int i = 0; i < B; ++i) {
      const int b = p.order[i];
      jobs[i] = (int64_t)row_tiles(seqs->suffix_len[b], G) * pool->num_kv_heads;
      kt[i] = ((int64_t)seqs->prefix_len[b] + seqs->suffix_len[b] + kvt::kExtKeysPerTile - 1) / kvt::kExtKeysPerTile;
    }
    auto cost = [&](int s) {
      double t = list_finish(0, 0.0, jobs, kt, s, xcd_cus, kXcds);
      if (s > 1) t += (2.0 * (double)part_bytes(pool, s, rows) / 5.0e6 + kMergeLaunchUs) / 1.8;
      return t;
    };
    const double rule_cost = cost(ns);
    int best = ns;
    double best_cost = rule_cost;
    for (int s = 1; s <= kvt::kMaxSplits; s *= 2) {
      const double c = cost(s);
      if (c < best_cost - 1e-9) best = s, best_cost = c;
    }
    if (best_cost < 0.8 * rule_cost) ns = best;
  }
  p.nsplit = p.nsplit_base = ns;
  if (ns > 1) p.ws_bytes = part_bytes(pool, ns, T * num_q_heads);
  return p;
}

// Weight of one key tile of the last row tile of a sequence against a full
// one's, by its waves that hold rows: up to four have a SIMD each to
// themselves (1.05 us per key tile with eight workgroups running, 1.42 to 1.63
// with all CUs busy on keys of their own), from five on they share SIMDs
// (1.41 to 1.50, 1.93 to 2.40).
constexpr double kTileWeight[3] = {0.65, 0.95, 1.0};
int last_tile_class(int32_t suffix, int group) {
  const int64_t rows = (int64_t)suffix * group % kvt::kExtTileRows;
  if (rows == 0) return 2;
  return rows <= 4 * kvt::kExtRowsPerWave ? 0 : 1;
}

// Key splits of a last row tile of one class: fewer than the full row tiles
// take when it is lighter, so that every unit takes about as long.
int last_splits(int nsplit, double heaviest, int tile_class) {
  if (heaviest == 0.0 || kTileWeight[tile_class] == heaviest) return nsplit;
  return std::max(1, (int)std::lround(nsplit * kTileWeight[tile_class] / heaviest));
}

// The split plan of an extend call is make_plan's, unless the call has at most
// one row tile per CU and like contexts (the longest at most twice the
// shortest): then refine_plan looks further.  make_plan counts every row tile
// as full and keeps 1024 keys per split, which leaves most of the chip idle for
// a short message over a few thousand keys; here the row tiles of one kv-head,
// each with its weight, are laid over that head's share of the CUs for a range
// of split counts (up to kMaxPartials, down to one key tile per split), every
// unit charged its key tiles, kUnitTiles, and every round of units in full, and
// the merge charged 4.5 us and its partials at 4.5 TB/s.  The best is taken if
// it beats make_plan's count by more than 5 %, and an unsplit one also by 6 key
// tiles (the second launch and the workspace cost the host about 5 us, the
// device a launch gap).  Plans whose partials would no longer fit the no-alloc
// entry point's static scratch where make_plan's do are left alone: one plan
// serves both entry points, and what the no-alloc one took it takes.  Per pass, make_plan's count and this one: 37 new tokens over 2000
// keys, 32/8 heads, 51.1 and 29.3 us; 64 over 131072, 24/2 heads, 196 and
// 113 us; 67 over 30011, 32/8 heads, 61.1 and 56.8 us; 20 over 700 keys (left
// alone) 24 and 29 us.
void refine_plan(ExtendPlan* p, const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads, int64_t T, int cus) {
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads;
  const int64_t rows = T * num_q_heads;
  const int longest = p->order.front(), shortest = p->order.back();
  const int64_t max_len = (int64_t)seqs->prefix_len[longest] + seqs->suffix_len[longest];
  const int64_t min_len = (int64_t)seqs->prefix_len[shortest] + seqs->suffix_len[shortest];
  const int head_cus = cus / pool->num_kv_heads;
  if (max_len > 2 * min_len || B > head_cus) return;
  int64_t tiles = 0;   // row tiles of one kv-head: full ones, and last ones by class
  int last[3] = {0, 0, 0};
  double heaviest = 0.0;
  for (int b = 0; b < B; ++b) {
    const int t = row_tiles(seqs->suffix_len[b], G), c = last_tile_class(seqs->suffix_len[b], G);
    tiles += t;
    ++last[c];
    heaviest = std::max(heaviest, t > 1 ? 1.0 : kTileWeight[c]);
  }
  if (tiles > head_cus) return;
  const int full = (int)tiles - B;
  const int kt = (int)((max_len + kvt::kExtKeysPerTile - 1) / kvt::kExtKeysPerTile);
  auto cost = [&](int ns, bool weighted) {
    int units = full * ns;   // at most 64 per CU
    for (int c = 0; c < 3; ++c)
      if (last[c] > 0) units += last[c] * (weighted ? last_splits(ns, heaviest, c) : ns);
    const double unit = heaviest * (double)((kt + ns - 1) / ns) + kUnitTiles;
    const double merge = ns > 1 ? (4.5 + (double)part_bytes(pool, ns, rows) / 4.5e6) / 1.8 : 0.0;
    return (double)((units + head_cus - 1) / head_cus) * unit + merge;
  };
  const double base = cost(p->nsplit, false);
  int best = 0;
  double best_cost = 0.95 * base - (p->nsplit == 1 ? 6.0 : 0.0);
  double per_split = (double)full;   // units per split count
  for (int b = 0; b < B; ++b) per_split += kTileWeight[last_tile_class(seqs->suffix_len[b], G)] / heaviest;
  auto consider = [&](int ns) {
    if (ns < 1 || ns > kvt::kMaxPartials || ns > kt) return;
    const double c = cost(ns, true);
    if (c < best_cost - 1e-9) best = ns, best_cost = c;
  };
  for (int ns = 1; ns <= kvt::kMaxPartials; ns *= 2) consider(ns);
  for (int r = 1; r <= 3; ++r)   // the counts that fill whole rounds (or just do, where rounding adds a unit)
    for (int ns = (int)(r * head_cus / per_split), k = 0; k < 2; ++k) consider(ns - k);
  if (best == 0) return;
  const size_t bytes = best > 1 ? part_bytes(pool, best, rows) : 0;
  if (bytes > (size_t)KVT_NOALLOC_SCRATCH_BYTES && p->ws_bytes <= (size_t)KVT_NOALLOC_SCRATCH_BYTES) return;
  p->nsplit = best;
  p->heaviest = heaviest;
  p->ws_bytes = bytes;
}

ExtendPlan extend_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads, int64_t T) {
  const int cus = device_cus();
  ExtendPlan p = make_plan(pool, seqs, num_q_heads, T, cus);
  refine_plan(&p, pool, seqs, num_q_heads, T, cus);
  return p;
}

// Keys of a decoding batch (each sequence's new one included).
int64_t total_keys(const kvt_seqs* seqs) {
  int64_t total = seqs->num_seqs;
  for (int b = 0; b < seqs->num_seqs; ++b) total += seqs->prefix_len[b];
  return total;
}

// Workgroups of a decode launch that share a CU: 0 for as many as fit (two with
// heads of 128; four with heads of 64, three in fp32), else fewer.  Where one
// has a CU to itself, units run longest first, each at the CU's full rate, and
// short ones fill the CUs that become free.  Where several share it, the first
// units share the bandwidth as well, and when the shorter ones have ended, the
// longest are too few to use it.  `reach` is how much of a step the longest
// unit takes at half a CU; `mean` is the mean unit's keys.
//   * Unlike contexts: one per CU from reach 1.05 on (from 1.5 on in split
//     plans of 3.5 and more units per CU; with bf16 heads of 64 in split plans
//     and below 3000 keys a unit), if units are long enough to hide a
//     workgroup's start and end without a neighbour (below that from 2.4 on).
//     Per step, two per CU and one, 96/8 heads of 128: 64 contexts of
//     1000..8192 keys (reach 2.6) 147.9, 129.8 us; 90 of 2000..32768 (2.4)
//     615.7, 537.2; 128 of 1000..8192 (1.3) 258.8, 256.3; 100 of 1000..8192 in
//     two splits (0.8) 219.1, 229.7; 32 of 2048..32768 in four (1.4) 242.0,
//     244.5; 48 in three (1.6) 279.0, 272.7; 28 of 13000..39800 in three (1.15,
//     672 units) 434.1, 413.7; 48 of 500..4096 in two (1.8, 850 keys a unit)
//     53.2, 57.5.  Otherwise at most two: 32/8 heads of 64, four and two: 160
//     of 1000..8192 158.2, 153.5; 128 of 500..4096 69.8, 65.0; but 256 of
//     100..600 31.8, 38.6.
//   * Like contexts fill whole rounds, so what the last round (of two per CU)
//     leaves decides: 90 of 4000..8000 keys (208 units in it) 341.9, 319.4 us;
//     48 in two splits (256) 188.3, 180.8; but 72 (64 units) 263.4, 273.0; 100
//     (288) 373.5, 383.2; 64 (none) 237.8, 230.6.  With four per CU, a last
//     round that is nearly full, or lengths that differ, in the first: heads of
//     64, four and two: 100 of 2000..4000 keys (800 units) 102.4, 94.5; 112 of
//     4000..8000 (896) 212.1, 206.3; 72 of 4000..8000 (reach 1.2) 145.4, 136.3;
//     but 72 of 4096 (0.9) 105.1, 119.6; 200 of 4000..8000 (576) 375.7, 388.0.
int decode_per_cu(const kvt_pool* pool, const kvt_seqs* seqs, const ExtendPlan& plan) {
  const int64_t cus = device_cus(), units = (int64_t)seqs->num_seqs * plan.nsplit * pool->num_kv_heads;
  if (units <= cus) return 0;
  const int64_t max_keys = (int64_t)seqs->prefix_len[plan.order.front()] + 1;
  const int64_t min_keys = (int64_t)seqs->prefix_len[plan.order.back()] + 1;
  const double longest = (double)max_keys / plan.nsplit;
  const double mean = (double)total_keys(seqs) / ((double)seqs->num_seqs * plan.nsplit);
  const double reach = 2.0 * longest / (mean * (double)units / (double)cus);
  if (max_keys > 2 * min_keys) {
    if (mean < 1500) return mean >= 800 && reach >= 2.4 ? 1 : 0;
    const bool late = pool->head_dim == 64 && pool->dtype == KVT_DTYPE_BF16
                          ? plan.nsplit > 1 || mean < 3000
                          : plan.nsplit > 1 && 2 * units >= 7 * cus;
    return reach >= (late ? 1.5 : 1.05) ? 1 : 2;
  }
  if (mean < 1500) return 0;
  if (pool->head_dim == 64) {
    if (pool->dtype != KVT_DTYPE_BF16) return 0;
    return units % (4 * cus) >= 3 * cus || (units < 4 * cus && reach >= 1.1) ? 2 : 0;
  }
  const int64_t rest = units % (2 * cus);
  return (rest == 0 && reach >= 1.35) || (2 * rest >= cus && rest <= cus && reach >= 0.9) ? 1 : 0;
}

// Decode: one unit per (sequence, key split) and kv-head.  Splits are added
// while the workgroups cannot cover the CUs twice over (two share a CU), at
// most kMaxSplits, keeping at least 1024 keys of the shortest sequence per
// split (each of the 4 waves then streams at least 8 tiles of 32 keys).
// Beside that base count:
//   * a small batch of like contexts (the longest at most twice the shortest)
//     would leave CUs idle; its splits fill the CUs once, down to 128 keys
//     per split (one tile per wave), at most kMaxPartials.  One context,
//     kernel + merge: 131072 keys of 8 kv-heads 98.3 + 4.3 us at 16 splits,
//     81.8 + 4.9 at 32 (256 workgroups), 88.2 + 7.5 at 64; 2048 keys 17.1 + 2.4
//     at 2, 9.6 + 2.6 at 8, 8.2 + 3.0 at 16.  Where the base count is 1 that
//     adds the merge, so the splits have to take 400 keys (heads of 64: 500)
//     from the longest workgroup: 8 kv-heads, unsplit and split, 16 contexts of
//     600 keys (2 splits) 12.6, 13.8 us, of 1300 20.8, 19.9; 8 of 600 (4) 12.2,
//     12.1, of 1000 16.0, 12.8; with heads of 64 16 of 600 8.3, 9.6, of 1300
//     12.9, 12.2.  In fp32 half the CUs already reach the bandwidth: two splits
//     of 16 contexts of 1700 keys 36.2, 39.5, heads of 64 19.5, 22.5;
//   * from one unit per CU on, if a unit of the longest context takes longer
//     than a CU's mean share of the keys, the longest contexts decide when the
//     step ends; with two rounds of workgroups (four per CU in all) and at
//     least 4096 keys of the longest per split, the rest fills in beside them.
//     So it does if like contexts leave a last round (of two per CU) nearly
//     empty, and in any batch where only one workgroup fits a CU (fp32 heads
//     of 128: 36 contexts of 2091..16734 keys 569 us at 2 splits, 550 at 4).
//     Per step of 32 contexts at 2, 3, 4, 6 splits: 2048..32768 keys 287, 260,
//     247, 251 us; 16384..32768 keys (the longest unit 0.7 of a CU's share)
//     497, 514, 490, 503 us; 64 contexts of 8192 keys (0.5) at 1 and 2: 325,
//     342 us; 70 (48 workgroups in the last round) 396, 383; 80 (128) 413, 428.
ExtendPlan make_decode_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  ExtendPlan p;
  const int B = seqs->num_seqs;
  p.order.resize(B);
  std::iota(p.order.begin(), p.order.end(), 0);
  std::stable_sort(p.order.begin(), p.order.end(),
                   [&](int x, int y) { return seqs->prefix_len[x] > seqs->prefix_len[y]; });
  const int64_t max_keys = (int64_t)seqs->prefix_len[p.order.front()] + 1;
  const int64_t min_keys = (int64_t)seqs->prefix_len[p.order.back()] + 1;
  const int64_t units = (int64_t)B * pool->num_kv_heads;
  const int64_t cus = device_cus();
  const bool like = max_keys <= 2 * min_keys;
  const int64_t want = (2 * cus + units - 1) / units;
  const int64_t by_keys = std::max<int64_t>(1, min_keys / 1024);
  p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>({want, by_keys, (int64_t)kvt::kMaxSplits}));
  p.nsplit_base = p.nsplit;
  if (like) {
    const int64_t fill = std::min<int64_t>({cus / units, min_keys / 128, (int64_t)kvt::kMaxPartials});
    const bool pays = max_keys * (fill - 1) >= (pool->head_dim == 64 ? 500 : 400) * fill &&
                      (fill > 2 || pool->dtype == KVT_DTYPE_BF16);
    if (p.nsplit > 1 || pays) p.nsplit = (int)std::max<int64_t>(p.nsplit, fill);
  }
  const int64_t rest = units * p.nsplit % (2 * cus);
  const bool one_fits = pool->dtype == KVT_DTYPE_F32 && pool->head_dim == 128;
  if (units >= cus && (one_fits || max_keys * cus >= total_keys(seqs) * pool->num_kv_heads * p.nsplit ||
                       (like && rest > 0 && 2 * rest < cus))) {
    const int64_t rounds = (4 * cus + units / 2) / units;   // to the nearest
    p.nsplit = (int)std::max<int64_t>(p.nsplit, std::min(rounds, max_keys / 4096));
  }
  if (p.nsplit > 1) p.ws_bytes = part_bytes(pool, p.nsplit, (int64_t)B * num_q_heads);
  return p;
}

// Fits a plan to the workspace a call offers: the plan itself when it fits,
// unsplit when none is offered, and else the base split count, which asks
// for no more than any call with these arguments ever had to offer: where it
// is unsplit, any workspace argument will do.
kvt_status fit_workspace(ExtendPlan* plan, const kvt_pool* pool, int64_t rows, const void* workspace,
                         size_t workspace_bytes) {
  if (plan->nsplit == 1) return KVT_OK;
  if (workspace == nullptr && workspace_bytes == 0) {
    plan->nsplit = 1;   // no scratch offered: run unsplit
    plan->heaviest = 0.0;
    return KVT_OK;
  }
  if (workspace != nullptr && workspace_bytes >= plan->ws_bytes && aligned16(workspace)) return KVT_OK;
  plan->nsplit = plan->nsplit_base;
  plan->heaviest = 0.0;
  if (plan->nsplit == 1) return KVT_OK;
  plan->ws_bytes = part_bytes(pool, plan->nsplit, rows);
  if (workspace == nullptr || workspace_bytes < plan->ws_bytes) return KVT_ERR_WORKSPACE;
  return aligned16(workspace) ? KVT_OK : KVT_ERR_INVALID_ARG;
}

// A shared prefix: a positive multiple of 16 no longer than any sequence's
// prefix; in checked mode every table row must list the same pages for it.
kvt_status check_shared(const kvt_seqs* seqs, int32_t shared_len) {
  if (shared_len < kvt::kBlock || shared_len % kvt::kBlock != 0) return KVT_ERR_INVALID_ARG;
  for (int b = 0; b < seqs->num_seqs; ++b)
    if (seqs->prefix_len[b] < shared_len) return KVT_ERR_INVALID_ARG;
  if (seqs->block_table_host != nullptr) {
    const int32_t* row0 = seqs->block_table_host;
    for (int b = 1; b < seqs->num_seqs; ++b)
      if (std::memcmp(row0, seqs->block_table_host + (int64_t)b * seqs->max_blocks,
                      sizeof(int32_t) * (shared_len / kvt::kBlock)) != 0)
        return KVT_ERR_INVALID_ARG;
  }
  return KVT_OK;
}

// Estimated time of one extend launch in units of one 64-key tile of one
// 256-row workgroup: the larger of the work spread over the CUs and the
// longest unit's share of its key splits, plus the split partials written
// and read back when split.
double launch_estimate(const kvt_seqs* seqs, int group, int kv_heads, int nsplit, int64_t rows, const kvt_pool* pool,
                       int cus) {
  // one tile of one workgroup takes about 1.8 us at full load; the partials
  // move at about 5 TB/s (written once, read once by the combine),
  // and the combine launch itself costs about 4 us
  constexpr double kTileUs = 1.8, kBytesPerUs = 5.0e6;
  double work = 0, longest = 0;
  for (int b = 0; b < seqs->num_seqs; ++b) {
    const int64_t kt = ((int64_t)seqs->prefix_len[b] + seqs->suffix_len[b] + kvt::kExtKeysPerTile - 1) /
                       kvt::kExtKeysPerTile;
    work += (double)((int64_t)row_tiles(seqs->suffix_len[b], group) * kv_heads) * kt;
    longest = std::max(longest, (double)kt);
  }
  double t = std::max(work / cus, longest / nsplit) + kUnitTiles;
  if (nsplit > 1) t += (2.0 * (double)part_bytes(pool, nsplit, rows) / kBytesPerUs + kMergeLaunchUs) / kTileUs;
  return t;
}

// Cascade: the split plans of the shared part (one virtual sequence of all T
// new tokens over the shared keys, all visible) and of the private parts
// (prefix lengths less the shared prefix); the workspace holds one partial
// per split of either part.  The shared pass reads the shared keys once per
// packed row tile of the whole batch instead of once per sequence's row
// tiles, but every row then goes through partials and a merge; when the
// estimate says the plain extend is faster (long suffixes, where row tiles
// pack well anyway), the plan is the plain extend's (use_shared = false).
//
// The choice is made with make_plan's split counts; the route that runs is then
// refined as a short message's plan is (refine_plan; the shared pass unless
// `base`, and if the estimate gains more than 5 %).  Host time of a plan: 4.5
// us for 24 forks on one kv-head, 2.7 for 16 on eight (26.3 and 18.7 with both
// routes refined and every unit through a heap of the CUs, 9.2 and 14.5 with
// that heap before there was anything to refine).
// 3 sequences adding 3..16 tokens over 4096 shared keys, 32/8 heads: 29.6 us per
// pass with make_plan's count, 25.7 with this; 9 adding 5..20, 24/2 heads, 40.0
// and 33.5.  Calls that fill the chip keep their count (16 over 32768 shared).
ExtendPlan cascade_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t shared_len, int32_t num_q_heads,
                        int64_t T, int32_t mode = KVT_CASCADE_AUTO, bool base = false) {
  if (mode == KVT_CASCADE_PLAIN) {
    ExtendPlan plain = extend_plan(pool, seqs, num_q_heads, T);
    plain.use_shared = false;
    return plain;
  }
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads, H = pool->num_kv_heads;
  const int KT = kvt::kExtKeysPerTile;
  const int cus = device_cus();
  const int64_t rows = T * num_q_heads;
  std::vector<int32_t> priv(B);
  for (int b = 0; b < B; ++b) priv[b] = seqs->prefix_len[b] - shared_len;
  kvt_seqs ps = *seqs;
  ps.prefix_len = priv.data();
  const int32_t shared_prefix = shared_len - 1, all_tokens = (int32_t)T;
  kvt_seqs ss = *seqs;
  ss.num_seqs = 1;
  ss.prefix_len = &shared_prefix;
  ss.suffix_len = &all_tokens;
  ExtendPlan shared_plan = make_plan(pool, &ss, num_q_heads, T, cus);

  int64_t head_jobs = 0;   // private units of one kv-head
  for (int b = 0; b < B; ++b) head_jobs += row_tiles(seqs->suffix_len[b], G);
  const int head_cus = std::max(1, cus / H);
  const bool one_round = head_jobs <= head_cus;
  ExtendPlan p;
  if (one_round) p.order = longest_first(&ps);   // the split count is placed below
  else p = make_plan(pool, &ps, num_q_heads, T, cus);
  std::vector<int64_t> jobs_p(B), kt_p(B);   // launch order, longest first; one kv-head's units
  for (int i = 0; i < B; ++i) {
    const int b = p.order[i];
    jobs_p[i] = row_tiles(seqs->suffix_len[b], G);
    kt_p[i] = ((int64_t)priv[b] + seqs->suffix_len[b] + KT - 1) / KT;
  }
  const int64_t shared_tiles = row_tiles((int32_t)T, G);
  const double kt_shared = (double)((shared_len + KT - 1) / KT);
  auto partial_cost = [&](int parts) {
    return (2.0 * (double)part_bytes(pool, parts, rows) / 5.0e6 + kMergeLaunchUs) / 1.8;
  };
  // Split counts of both parts with ns_s splits of the shared part, and their
  // estimate.  In one launch the private units can fill what the shared part
  // leaves idle: when one kv-head's private units fit one round of its CUs,
  // their split count is the one (trying 1, 2, 4, 8, 16 until the estimate
  // rises) with the earliest list-scheduled finish plus partial cost.
  auto place = [&](int ns_s, int* ns_p) {
    const int64_t head_shared = shared_tiles * ns_s;
    const double len_s = std::ceil(kt_shared / ns_s);
    if (one_round) {
      int best = 1;
      double t = list_finish(head_shared, len_s, jobs_p, kt_p, 1, head_cus) + partial_cost(ns_s + 1);
      for (int ns = 2; ns <= kvt::kMaxSplits; ns *= 2) {
        const double c = list_finish(head_shared, len_s, jobs_p, kt_p, ns, head_cus) + partial_cost(ns_s + ns);
        if (c >= t - 1e-9) break;
        best = ns, t = c;
      }
      *ns_p = best;
      return t;
    }
    // many private units: the work of both parts spread over the CUs, or
    // the longest unit of either
    double work = (double)(head_shared * H) * len_s, longest = len_s;
    for (int i = 0; i < B; ++i) {
      work += (double)(jobs_p[i] * H) * kt_p[i];
      longest = std::max(longest, (double)kt_p[i] / p.nsplit);
    }
    *ns_p = p.nsplit;
    return std::max(work / cus, longest) + kUnitTiles + partial_cost(ns_s + p.nsplit);
  };
  int ns_p = 1;
  const double t_shared = place(shared_plan.nsplit, &ns_p);

  if (mode == KVT_CASCADE_AUTO) {
    // the choice weighs make_plan's split counts, whatever refine_plan makes of them
    ExtendPlan plain = make_plan(pool, seqs, num_q_heads, T, cus);
    if (!(t_shared < launch_estimate(seqs, G, H, plain.nsplit, rows, pool, cus))) {
      refine_plan(&plain, pool, seqs, num_q_heads, T, cus);
      plain.use_shared = false;
      return plain;
    }
  }
  int ns_s = shared_plan.nsplit;
  if (!base) {
    refine_plan(&shared_plan, pool, &ss, num_q_heads, T, cus);
    const int ns = std::min(shared_plan.nsplit, kvt::kMaxPartials - kvt::kMaxSplits);
    // the shared units alone, with one private set, are a lower bound: place
    // nothing when even they gain too little
    const double len = std::ceil(kt_shared / ns);
    const double least = one_round ? (double)((shared_tiles * ns + head_cus - 1) / head_cus) * (len + kUnitTiles)
                                   : len + kUnitTiles;
    int q = 1;
    if (ns != ns_s && least + partial_cost(ns + 1) < 0.95 * t_shared && place(ns, &q) < 0.95 * t_shared)
      ns_s = ns, ns_p = q;
  }
  p.nsplit_shared = ns_s;
  p.nsplit = ns_p;
  p.ws_bytes = part_bytes(pool, ns_s + ns_p, rows);
  return p;
}

bool mode_ok(int32_t mode) {
  return mode == KVT_CASCADE_AUTO || mode == KVT_CASCADE_SHARED_PASS || mode == KVT_CASCADE_PLAIN;
}

// out must not overlap q or a pool; lse must not overlap out.
kvt_status check_outputs(const kvt_pool* pool, const void* q, int32_t num_q_heads, const void* out,
                         const float* lse, int64_t T, bool mx = false) {
  if (!aligned16(q) || !aligned16(out) || ((uintptr_t)lse & 3) != 0) return KVT_ERR_INVALID_ARG;
  const size_t es = elem_bytes(pool->dtype);
  const size_t tok_bytes = (size_t)T * num_q_heads * pool->head_dim * es;
  const size_t pool_bytes = pool_tensor_bytes(pool, mx);
  if (overlaps(out, tok_bytes, q, tok_bytes) || overlaps(out, tok_bytes, pool->k, pool_bytes) ||
      overlaps(out, tok_bytes, pool->v, pool_bytes))
    return KVT_ERR_INVALID_ARG;
  if (lse != nullptr && overlaps(lse, (size_t)T * num_q_heads * sizeof(float), out, tok_bytes))
    return KVT_ERR_INVALID_ARG;
  return KVT_OK;
}

// Launch arguments common to extend and decode.
kvt::ExtendArgs base_args(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                          float scale, void* out, float* lse, int64_t T, const ExtendPlan& plan, void* workspace) {
  kvt::ExtendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.out = out;
  a.lse = lse;
  a.block_table = seqs->block_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = pool->num_kv_heads;
  a.group = num_q_heads / pool->num_kv_heads;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.kbeg = 0;
  a.kend = INT32_MAX;
  a.direct = plan.nsplit == 1 ? 1 : 0;
  a.part_base = 0;
  a.nsplit = plan.nsplit;
  a.total_rows = (int32_t)T;
  a.second = INT32_MAX;   // one group of sequences
  a.kbeg2 = 0;
  a.kend2 = INT32_MAX;
  a.nsplit2 = 1;
  a.part_base2 = 0;
  if (plan.nsplit > 1) {
    a.part_o = reinterpret_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) +
                                         part_o_bytes(pool, plan.nsplit, T * num_q_heads));
  }
  return a;
}

// Merge of the per-split partial results into out (and lse).
kvt_status combine(const kvt::ExtendArgs& a, const kvt_pool* pool, void* out, float* lse, int64_t T,
                   int32_t num_q_heads, int nsplit, bool gaps, hipStream_t s) {
  kvt::CombineArgs c;
  c.part_o = a.part_o;
  c.part_ml = a.part_ml;
  c.out = out;
  c.lse = lse;
  c.rows = T * num_q_heads;
  c.nsplit = nsplit;
  c.gaps = gaps ? 1 : 0;
  const hipError_t e = kvt::launch_combine(c, pool->dtype, pool->head_dim, s);
  return e == hipSuccess ? KVT_OK : device_error(e);
}

// Per-token rows of `width` elements of `es` bytes: where the `T` rows lie.
struct Rows {
  uintptr_t first;
  size_t width, step;   // bytes of a row, bytes from row to row
  int64_t n;
  size_t extent() const { return (size_t)(n - 1) * step + width; }
};
kvt_status check_rows(const kvt_rows* r, int64_t T, int64_t width, int es, Rows* out) {
  if (r->data == nullptr || !aligned16(r->data)) return KVT_ERR_INVALID_ARG;
  const int64_t stride = T == 1 ? width : r->stride;
  if (stride < width || stride * es % 16 != 0 || stride > INT64_MAX / 8 / T) return KVT_ERR_INVALID_ARG;
  *out = Rows{(uintptr_t)r->data, (size_t)(width * es), (size_t)(stride * es), T};
  return KVT_OK;
}
// Whether two row sets share a byte.  Rows of one stride interleave without
// touching (parts of one fused projection); of two strides only disjoint
// extents are taken as apart.
bool rows_touch(const Rows& x, const Rows& y) {
  if (!overlaps((const void*)x.first, x.extent(), (const void*)y.first, y.extent())) return false;
  if (x.step != y.step) return true;
  const size_t ahead = y.first >= x.first ? (y.first - x.first) % x.step
                                          : (x.step - (x.first - y.first) % x.step) % x.step;
  return ahead < x.width || ahead + y.width > x.step;
}
bool rows_same(const Rows& x, const Rows& y) { return x.first == y.first && x.width == y.width && x.step == y.step; }

// Whether rows that a call writes reach into the positions that it reads.
bool covers_positions(const Rows& out, const kvt_rotary* r) {
  return r->positions != nullptr && overlaps((const void*)out.first, out.extent(), r->positions,
                                             (size_t)r->num_axes * out.n * sizeof(int32_t));
}

// The rotary description; fills the launch's frequencies.
kvt_status check_rotary(const kvt_rotary* r, int32_t head_dim, kvt::RotaryArgs* a) {
  if (r == nullptr || r->inv_freq == nullptr) return KVT_ERR_INVALID_ARG;
  if ((r->parts != 1 && r->parts != 2) || (r->interleaved != 0 && r->interleaved != 1)) return KVT_ERR_INVALID_ARG;
  if (r->rot_dim < 16 || r->rot_dim % 16 != 0 || r->rot_dim > head_dim / r->parts) return KVT_ERR_INVALID_ARG;
  if (r->num_axes < 1 || r->num_axes > 64) return KVT_ERR_INVALID_ARG;
  if (((uintptr_t)r->positions & 3) != 0) return KVT_ERR_INVALID_ARG;
  for (int j = 0; j < r->rot_dim / 2; ++j) {
    if (!std::isfinite(r->inv_freq[j])) return KVT_ERR_INVALID_ARG;
    const int32_t axis = r->axis != nullptr ? r->axis[j] : 0;
    if (axis < 0 || axis >= r->num_axes) return KVT_ERR_INVALID_ARG;
    a->turns[j] = (double)r->inv_freq[j] / (2.0 * 3.14159265358979323846);
    a->axis[j] = (uint8_t)axis;
  }
  a->positions = r->positions;
  a->rot_dim = r->rot_dim;
  a->parts = r->parts;
  a->interleaved = r->interleaved;
  return KVT_OK;
}

// The argument checks of kvt_extend_attention (and its no-alloc variant);
// fills the total token count.
kvt_status check_extend(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads, float scale,
                        const void* out, const float* lse, int64_t* T, bool mx = false) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  if ((st = check_seqs(seqs, T)) != KVT_OK) return st;
  if (q == nullptr || out == nullptr) return KVT_ERR_INVALID_ARG;
  if (!heads_ok(pool, num_q_heads, *T)) return KVT_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  return check_outputs(pool, q, num_q_heads, out, lse, *T, mx);
}

// Launches of one extend call under `plan` (partials in `workspace` when split);
// `mx`: over 4-bit pages.
kvt_status launch_extend_plan(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                              float scale, void* out, float* lse, int64_t T, const ExtendPlan& plan,
                              void* workspace, void* stream, bool mx = false) {
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int G = num_q_heads / pool->num_kv_heads;
  std::vector<int32_t> row_off(seqs->num_seqs + 1, 0);
  for (int b = 0; b < seqs->num_seqs; ++b) row_off[b + 1] = row_off[b] + seqs->suffix_len[b];

  kvt::ExtendArgs a = base_args(pool, seqs, q, num_q_heads, scale, out, lse, T, plan, workspace);
  for (size_t c0 = 0; c0 < plan.order.size(); c0 += kvt::kSeqsPerLaunch) {
    const int n = (int)std::min<size_t>(kvt::kSeqsPerLaunch, plan.order.size() - c0);
    a.nseq = n;
    int32_t units = 0;
    for (int i = 0; i < n; ++i) {
      const int b = plan.order[c0 + i];
      const int last = last_splits(plan.nsplit, plan.heaviest, last_tile_class(seqs->suffix_len[b], G));
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row_off[b]};
      a.last[i] = (uint8_t)last;
      a.unit_begin[i] = units;
      units += (row_tiles(seqs->suffix_len[b], G) - 1) * plan.nsplit + last;
    }
    a.unit_begin[n] = units;
    const int64_t grid = (int64_t)units * pool->num_kv_heads;
    if (grid > INT32_MAX) return KVT_ERR_INVALID_ARG;
    const hipError_t e = mx ? kvt::launch_mx_extend(a, pool->dtype, pool->head_dim, (int)grid, s)
                             : kvt::launch_extend(a, pool->dtype, pool->head_dim, (int)grid, s);
    if (e != hipSuccess) return device_error(e);
  }
  return plan.nsplit > 1 ? combine(a, pool, out, lse, T, num_q_heads, plan.nsplit, plan.heaviest > 0.0, s) : KVT_OK;
}

// Key splits of a differential attention call: every sequence has its own
// count, so that long contexts split beside short ones that do not, and the
// partial rows of the split ones lie one after the other.
struct DiffPlan {
  std::vector<int> order;          // sequences, longest key range first
  std::vector<int32_t> nsplit;     // by sequence
  std::vector<int32_t> nlast;      // by sequence: of its last row tile (extend)
  std::vector<int32_t> part_row;   // by sequence: first partial row (0 where it is not split)
  int64_t part_rows = 0;
  size_t ws_bytes = 0;
  bool one_per_cu = false;         // decode: workgroups that do not share a CU
};

size_t diff_o_bytes(const kvt_pool* pool, int64_t part_rows) {
  return ((size_t)part_rows * 2 * pool->head_dim * sizeof(float) + 255) / 256 * 256;
}

// Lays out the partial rows of the plan's splits; more than 32-bit row indices
// hold (terabytes of them) runs unsplit.
void diff_layout(DiffPlan* p, const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  const int B = seqs->num_seqs;
  p->part_row.assign(B, 0);
  p->part_rows = 0;
  for (int b = 0; b < B; ++b) {
    if (p->nsplit[b] == 1) continue;
    p->part_row[b] = (int32_t)p->part_rows;
    p->part_rows += (int64_t)p->nsplit[b] * seqs->suffix_len[b] * num_q_heads;
    if (p->part_rows > INT32_MAX) {
      p->nsplit.assign(B, 1);
      p->nlast.assign(B, 1);
      p->part_row.assign(B, 0);
      p->part_rows = 0;
      break;
    }
  }
  p->ws_bytes = p->part_rows > 0 ? diff_o_bytes(pool, p->part_rows) + (size_t)p->part_rows * 4 * sizeof(float) : 0;
}

int diff_row_tiles(int32_t suffix, int group) {
  return (int)(((int64_t)suffix * group + kvt::kDiffTileRows - 1) / kvt::kDiffTileRows);
}

// The splits of a differential extend call.  Every sequence's keys are cut into
// chunks of about equal length, the longest one's range divided by k, for a
// range of k; each k is charged the finish of its units (list scheduling, longest
// first, one XCD's eighth of the units on its CUs; with many sequences the work
// spread over the CUs and half a unit) and the merge: its partials at 4.5 TB/s and
// a launch.  The best k is taken if it beats no split by more than 5 %.  Times are
// in tiles of 64 keys: 1.69 us each with a few busy CUs, 2.15 with all (heads of
// 128, bf16; of 64 1.36 and 1.45), 11 us in fp32 (of 64 5.5).  bf16 heads of 64 run
// two units to a CU, together at 1.15 of one's rate (1024 new tokens over 16384, 32/8
// heads: unsplit 415 us, 2 splits 377; 512 over 8192: 2 splits 115 us, 4 110).
//
// A last row tile of up to 64 rows has a wave per SIMD and takes 0.63 (few busy CUs)
// to 0.65 (all) of a tile's time (fp32 0.53); beside full ones it gets as many splits
// less (67 over 30011, 32/8 heads of 128, charged with 0.66 of it 99.0 us, with 0.76
// 101.4).
DiffPlan diff_extend_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  DiffPlan p;
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads, H = pool->num_kv_heads;
  const int cus = device_cus(), KT = 64;
  p.order = longest_first(seqs);
  p.nsplit.assign(B, 1);
  const bool pairs = pool->dtype == KVT_DTYPE_BF16 && pool->head_dim == 64;
  const double both = pairs ? 1.15 : 1.0;   // rate of a CU with two units
  const double tile_us = pool->dtype != KVT_DTYPE_BF16 ? 11.0 * pool->head_dim / 128 : pool->head_dim == 64 ? 1.4 : 1.9;
  const double light = pool->dtype == KVT_DTYPE_BF16 ? 0.66 : 0.53;
  std::vector<int64_t> jobs(B), kt(B);   // jobs: full row tiles of all kv-heads
  std::vector<uint8_t> rest(B);          // whether a light one follows
  for (int i = 0; i < B; ++i) {
    const int b = p.order[i];
    const int tiles = diff_row_tiles(seqs->suffix_len[b], G);
    rest[i] = (int64_t)seqs->suffix_len[b] * G - (int64_t)(tiles - 1) * kvt::kDiffTileRows <= kvt::kDiffTileRows / 2;
    jobs[i] = (int64_t)(tiles - rest[i]) * H;
    kt[i] = ((int64_t)seqs->prefix_len[b] + seqs->suffix_len[b] + KT - 1) / KT;
  }
  constexpr int kXcds = 8, kListed = 32;
  const int xcd_cus = std::max(1, cus / kXcds);
  auto splits = [&](int i, int64_t chunk) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(kvt::kMaxPartials, (kt[i] + chunk - 1) / chunk));
  };
  auto light_splits = [&](int i, int ns) {
    return rest[i] && jobs[i] > 0 ? std::max(1, (int)std::ceil(light * ns)) : ns;
  };
  auto cost = [&](int64_t chunk) {
    double span = 0.0, work = 0.0, longest = 0.0, rows = 0.0;
    FreeTimes free_at(0.0, xcd_cus, 0.0, 0);
    auto put = [&](int64_t units, double len) {
      if (B <= kListed) span = std::max(span, free_at.run((units + kXcds - 1) / kXcds, len));
      work += (double)units * len;
      longest = std::max(longest, len);
    };
    for (int i = 0; i < B; ++i) {
      const int ns = splits(i, chunk), nl = light_splits(i, ns);
      if (jobs[i] > 0) put(jobs[i] * ns, std::ceil((double)kt[i] / ns) + kUnitTiles);
      if (rest[i]) put((int64_t)H * nl, light * (std::ceil((double)kt[i] / nl) + kUnitTiles));
      if (ns > 1) rows += (double)ns * seqs->suffix_len[p.order[i]] * num_q_heads;
    }
    if (B > kListed) span = std::max(longest, work / cus + 0.5 * longest);
    span = std::max(longest, span / both);
    return span + (rows > 0 ? (4.0 + 2.0 * rows * 2 * pool->head_dim * 4 / 4.5e6) / tile_us : 0.0);
  };
  int64_t best = kt[0];
  double best_cost = 0.95 * cost(kt[0]);
  for (int k : {2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16, 18, 20, 22, 24, 26, 28, 30, 32, 36, 40, 48, 64}) {
    if (k > kt[0]) break;
    if (B > 8 && k > 8 && k % 4 != 0) continue;   // large batches: fewer, for the host's sake
    const int64_t chunk = (kt[0] + k - 1) / k;
    const double c = cost(chunk);
    if (c < best_cost - 1e-9) best = chunk, best_cost = c;
  }
  p.nlast.assign(B, 1);
  for (int i = 0; i < B && best != kt[0]; ++i) {
    const int ns = splits(i, best);
    p.nsplit[p.order[i]] = ns;
    p.nlast[p.order[i]] = light_splits(i, ns);
  }
  diff_layout(&p, pool, seqs, num_q_heads);
  return p;
}

// The splits of a differential decoding step.  Every sequence is cut into chunks
// of about equal length (the nearest whole number of them), the chunk being one of
// a few fractions of a CU's share of all keys.  Each is charged the time in which
// the CUs, given the units longest first, stream them: one workgroup reads at up
// to 59 GB/s (heads of 64: 42; fp32: 25), all of them at 6.7 TB/s (fp32: 5.4), a
// unit's start and end count as 150 KB; and the joining launch, 4.5 us and its
// partials at 4.5 TB/s.  A cut has to gain 3 %.  Batches whose longest context is
// under half of a CU's share stay unsplit (192 of 1024..4096 keys).  Per step,
// unsplit and as chosen, heads of 128: one context of 131072 keys, 96/8 heads,
// 1126 and 87.5 us; 64 of 1024..16384, 96/8, 276 and 249; 8 of 2000..8000, 32/8,
// 73.5 and 31; 40 of 8000 (320 units on 256 CUs) 235 and 209.
//
// Unlike contexts in long units run one workgroup per CU (one_per_cu): where two
// share one, the longest get half its rate while the rest still runs (64 of
// 1024..16384 keys 256 and 249 us, 90 of 2000..32768 672 and 612); with many
// short units two hide each other's start and end (192 of 1024..4096 269.7 and
// 275; 100 of 200 keys 19.7 and 27).
DiffPlan diff_decode_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  DiffPlan p;
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads;
  const int64_t heads = (int64_t)pool->num_kv_heads * ((G + kvt::kDiffDecHeads - 1) / kvt::kDiffDecHeads);
  p.order = longest_first(seqs);
  p.nsplit.assign(B, 1);
  const int64_t longest = (int64_t)seqs->prefix_len[p.order.front()] + 1;
  const int64_t shortest = (int64_t)seqs->prefix_len[p.order.back()] + 1;
  const int64_t cus = device_cus(), all = total_keys(seqs) * heads;
  const bool bf16 = pool->dtype == KVT_DTYPE_BF16;
  auto splits = [&](int b, int64_t chunk) {
    const int64_t n = ((int64_t)seqs->prefix_len[b] + 1 + chunk / 2) / chunk;
    return (int)std::max<int64_t>(1, std::min<int64_t>(kvt::kMaxPartials, n));
  };
  int64_t chunk = 2 * longest;   // unsplit
  if (2 * longest * cus >= all) {
    const double key_bytes = 2.0 * pool->head_dim * elem_bytes(pool->dtype);
    const double one = !bf16 ? 25e3 : pool->head_dim == 64 ? 42e3 : 59e3, every = bf16 ? 6.7e6 : 5.4e6;   // bytes per us
    auto cost = [&](int64_t c) {
      FreeTimes cu(0.0, cus, 0.0, 0);
      double rows = 0;
      for (int i = 0; i < B; ++i) {
        const int b = p.order[i], n = splits(b, c);
        cu.run(n * heads, std::ceil((double)(seqs->prefix_len[b] + 1) / n) * key_bytes + 150e3);
        if (n > 1) rows += (double)n * num_q_heads;
      }
      return cu.drain(one, every) + (rows > 0 ? 4.5 + 2.0 * rows * 2 * pool->head_dim * 4 / 4.5e6 : 0.0);
    };
    double best = 0.97 * cost(chunk);
    for (double f : {0.7, 1.0, 1.5, 2.0, 3.0, 4.0}) {   // units per CU
      if (B > 32 && f != 1.0 && f != 1.5 && f != 3.0) continue;   // large batches: fewer, for the host's sake
      const int64_t c = std::max<int64_t>(128, (int64_t)((double)all / (f * (double)cus)));
      if (splits(p.order.front(), c) == 1) continue;
      const double t = cost(c);
      if (t < best) best = t, chunk = c;
    }
  }
  int64_t units = 0;
  for (int b = 0; b < B; ++b) units += (p.nsplit[b] = splits(b, chunk)) * heads;
  p.nlast = p.nsplit;
  const int64_t unit = (longest + p.nsplit[p.order.front()] - 1) / p.nsplit[p.order.front()];   // the longest one
  p.one_per_cu = units > cus && longest > 2 * shortest && all >= 1500 * units && 40 * unit * cus >= 21 * all;
  diff_layout(&p, pool, seqs, num_q_heads);
  return p;
}

size_t diff_lambda_bytes(const kvt_diff* diff, int32_t num_q_heads, int64_t T) {
  return ((size_t)(T - 1) * diff->lambda_stride + num_q_heads) * sizeof(float);
}

// The checks of both differential attention calls; fills the total token count.
kvt_status check_diff(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads, float scale,
                      const kvt_diff* diff, const void* out, int64_t* T) {
  kvt_status st = check_extend(pool, seqs, q, num_q_heads, scale, out, nullptr, T);
  if (st != KVT_OK) return st;
  if (diff == nullptr || diff->lambda == nullptr || ((uintptr_t)diff->lambda & 3) != 0) return KVT_ERR_INVALID_ARG;
  if (diff->lambda_stride != 0 &&
      (diff->lambda_stride < num_q_heads || diff->lambda_stride > INT64_MAX / 8 / *T))
    return KVT_ERR_INVALID_ARG;
  if (!std::isfinite(diff->out_scale)) return KVT_ERR_INVALID_ARG;
  const size_t out_bytes = (size_t)*T * num_q_heads * pool->head_dim * elem_bytes(pool->dtype);
  if (overlaps(out, out_bytes, diff->lambda, diff_lambda_bytes(diff, num_q_heads, *T))) return KVT_ERR_INVALID_ARG;
  if (diff->norm_weight != nullptr) {
    if (!aligned16(diff->norm_weight) || !(diff->eps > 0.f) || !std::isfinite(diff->eps)) return KVT_ERR_INVALID_ARG;
    if (overlaps(out, out_bytes, diff->norm_weight, pool->head_dim * sizeof(float))) return KVT_ERR_INVALID_ARG;
  }
  return KVT_OK;
}

// Launches of one differential attention call: the units of every sequence,
// then the join of those that are split.
kvt_status launch_diff(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads, float scale,
                       const kvt_diff* diff, void* out, int64_t T, DiffPlan& plan, bool decode, void* workspace,
                       size_t workspace_bytes, void* stream) {
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads;
  if (plan.ws_bytes > 0) {
    if (workspace == nullptr && workspace_bytes == 0) {   // no scratch offered: run unsplit
      plan.nsplit.assign(B, 1);
      plan.nlast.assign(B, 1);
      plan.ws_bytes = 0;
    } else {
      if (workspace == nullptr || workspace_bytes < plan.ws_bytes) return KVT_ERR_WORKSPACE;
      if (!aligned16(workspace)) return KVT_ERR_INVALID_ARG;
      const size_t io = (size_t)T * num_q_heads * pool->head_dim * elem_bytes(pool->dtype);
      if (overlaps(workspace, plan.ws_bytes, q, io) || overlaps(workspace, plan.ws_bytes, out, io) ||
          overlaps(workspace, plan.ws_bytes, diff->lambda, diff_lambda_bytes(diff, num_q_heads, T)) ||
          (diff->norm_weight != nullptr &&
           overlaps(workspace, plan.ws_bytes, diff->norm_weight, pool->head_dim * sizeof(float))))
        return KVT_ERR_INVALID_ARG;
    }
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  std::vector<int32_t> row_off(B + 1, 0);
  for (int b = 0; b < B; ++b) row_off[b + 1] = row_off[b] + seqs->suffix_len[b];
  kvt::DiffArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.out = out;
  a.lambda = diff->lambda;
  a.lambda_stride = diff->lambda_stride;
  a.norm_weight = diff->norm_weight;
  a.eps = diff->eps;
  a.out_scale = diff->out_scale;
  a.block_table = seqs->block_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = pool->num_kv_heads;
  a.group = G;
  a.scale_log2 = scale * 1.4426950408889634f;
  if (plan.ws_bytes > 0) {
    a.part_o = reinterpret_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + diff_o_bytes(pool, plan.part_rows));
  }
  auto describe = [&](int i, int b) {
    a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row_off[b]};
    a.nsplit[i] = (uint8_t)plan.nsplit[b];
    a.nlast[i] = (uint8_t)plan.nlast[b];
    a.part_row[i] = plan.part_row[b];
  };
  const int64_t per_unit = (int64_t)pool->num_kv_heads *
                           (decode ? (G + kvt::kDiffDecHeads - 1) / kvt::kDiffDecHeads : 1);   // workgroups
  for (int c0 = 0; c0 < B; c0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, B - c0);
    int64_t units = 0;
    for (int i = 0; i < n; ++i) {
      const int b = plan.order[c0 + i];
      describe(i, b);
      a.unit_begin[i] = (int32_t)units;
      units += (decode ? 0 : (int64_t)diff_row_tiles(seqs->suffix_len[b], G) - 1) * plan.nsplit[b] + plan.nlast[b];
      if (units * per_unit > INT32_MAX) return KVT_ERR_INVALID_ARG;
    }
    a.nseq = n;
    a.unit_begin[n] = (int32_t)units;
    const int grid = (int)(units * per_unit);
    const hipError_t e = decode ? kvt::launch_diff_decode(a, pool->dtype, pool->head_dim, grid, plan.one_per_cu, s)
                                : kvt::launch_diff_extend(a, pool->dtype, pool->head_dim, grid, s);
    if (e != hipSuccess) return device_error(e);
  }
  for (int c0 = 0; c0 < B && plan.ws_bytes > 0;) {
    int n = 0;
    int64_t rows = 0;
    for (; c0 < B && n < kvt::kSeqsPerLaunch; ++c0) {
      const int b = plan.order[c0];
      if (plan.nsplit[b] == 1) continue;
      describe(n, b);
      a.unit_begin[n++] = (int32_t)rows;
      rows += (int64_t)seqs->suffix_len[b] * num_q_heads;
    }
    if (n == 0) break;
    a.nseq = n;
    a.unit_begin[n] = (int32_t)rows;
    const hipError_t e = kvt::launch_diff_combine(a, pool->dtype, pool->head_dim, s);
    if (e != hipSuccess) return device_error(e);
  }
  return KVT_OK;
}

// ---- 4-bit pages and eviction

// The workspace of a call may not hold anything that the call reads or writes
// otherwise.
bool workspace_apart(const kvt_pool* pool, const void* q, const void* out, const float* lse, int32_t num_q_heads,
                     int64_t T, const void* workspace, size_t bytes) {
  const size_t io = (size_t)T * num_q_heads * pool->head_dim * elem_bytes(pool->dtype);
  const size_t held = pool_tensor_bytes(pool, true);
  return !overlaps(workspace, bytes, q, io) && !overlaps(workspace, bytes, out, io) &&
         !overlaps(workspace, bytes, pool->k, held) && !overlaps(workspace, bytes, pool->v, held) &&
         (lse == nullptr || !overlaps(workspace, bytes, lse, (size_t)T * num_q_heads * sizeof(float)));
}

// A call of few query rows over 4-bit pages (a decoding step, short chunks), launch
// by launch: see MxDecodeArgs.
struct MxDecodePlan {
  std::vector<int> order;          // sequences, longest key range first
  std::vector<int32_t> share;      // by launch: tiles of a slot, 0: slot x is sequence x
  std::vector<int32_t> parts;      // by place in `order`: slots that hold a part of the sequence
  std::vector<int32_t> chunks;     // by launch: workgroups that share the rows of a kv-head, of its largest message
  int64_t part_rows = 0;
  size_t ws_bytes = 0;
};

int64_t mx_tiles(const kvt_seqs* seqs, int b) {
  return ((int64_t)seqs->prefix_len[b] + seqs->suffix_len[b] + kvt::kDecKeysPerTile - 1) / kvt::kDecKeysPerTile;
}
bool mx_few_rows(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  for (int b = 0; b < seqs->num_seqs; ++b)
    if ((int64_t)seqs->suffix_len[b] * (num_q_heads / pool->num_kv_heads) > kvt::kMxFewRows) return false;
  return true;
}
size_t mx_part_o_bytes(const kvt_pool* pool, int64_t part_rows) {
  return ((size_t)part_rows * pool->head_dim * sizeof(float) + 255) / 256 * 256;
}

// What the choice below goes by, in us and bytes per us: a tile of a workgroup, more
// of it while another one runs on the CU; the stream of all workgroups, and of one to
// a CU; the join; a merge where a share goes on.  Messages of more than 16 rows run
// an instance with twice the products and exponentials.
struct MxRates {
  double tile, beside, stream, one, join, merge;
};
const MxRates& mx_rates(int head_dim, bool message) {
  static constexpr MxRates kRates[2][2] = {
      {{0.15, 0.12, 3.7e6, 2.9e6, 6.5, 1.5}, {0.30, 0.10, 2.3e6, 2.3e6, 10.0, 10.0}},
      {{0.18, 0.12, 5.5e6, 4.3e6, 6.5, 1.5}, {0.30, 0.10, 3.0e6, 3.0e6, 10.0, 10.0}}};
  return kRates[head_dim == 128 ? 1 : 0][message ? 1 : 0];
}

MxDecodePlan mx_decode_plan(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  MxDecodePlan p;
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads;
  p.order = longest_first(seqs);
  p.parts.assign(B, 1);
  const int64_t hkv = pool->num_kv_heads, cus = device_cus();
  for (int c0 = 0; c0 < B; c0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, B - c0);
    // tiles; those that the chunks with rows go through (a chunk past a sequence's
    // rows passes over it); chunks with rows
    int64_t total = 0, work = 0, chunks = 0, most = 1, rows = 0, longest_message = 0;
    for (int i = 0; i < n; ++i) {
      const int b = p.order[c0 + i];
      const int64_t of = ((int64_t)seqs->suffix_len[b] * G + kvt::kMxChunkRows - 1) / kvt::kMxChunkRows;
      total += mx_tiles(seqs, b);
      work += mx_tiles(seqs, b) * of;
      chunks += of;
      most = std::max(most, of);
      rows = std::max(rows, (int64_t)seqs->suffix_len[b] * G);
      longest_message = std::max<int64_t>(longest_message, seqs->suffix_len[b]);
    }
    p.chunks.push_back((int32_t)most);
    const int64_t longest = mx_tiles(seqs, p.order[c0]);
    // two workgroups to a CU, of at least 16 tiles (four for each wave).  One context
    // of 131072 keys and 64 of 1024..16384, 96/8 heads of 128, with one, two and
    // four: 41.0, 33.4 and 33.4 us, 107, 84 and 90
    const int64_t slots = std::max<int64_t>(1, 2 * cus * total / (hkv * work));
    int64_t share = std::max<int64_t>(16, (total + slots - 1) / slots);
    // a sequence lies in at most one slot more than its tiles fill
    share = std::max(share, (longest + kvt::kMxMaxParts - 2) / (kvt::kMxMaxParts - 1));
    // A slot for each sequence needs no join (a launch, the workspace) and no merge
    // where a share goes on to the next sequence.  A workgroup takes so long for a
    // tile, longer while another one runs on its CU; all of them stream so much, less
    // with one to a CU; and the shortest sequence starts last.  Steps of 32/8 heads of
    // 128, bf16, so and in shares: one context of 1000, 2000 and 3000 keys 11.1, 15.8
    // and 21.7 us, 16.5; 200 of 500..3000 62.9, 74.0 (16/2 heads 25.6, 31.5); 256 of
    // 100..600 28.2, 38.8; 100 of 1024..16384 131.8, 121.7; 70 of 6000 109.1, 87.5
    // (4/4 heads 60.3, 47.3); 100 of 500..3000 38.7, 47.1, heads of 64 28.3, 37.2, with
    // fp32 queries 27.9, 43.4.  The rates are from 1464 calls timed both ways (heads of
    // 64 and 128, bf16 and fp32, single tokens and messages, 1 to 200 contexts of 300 to
    // 131000 keys): the choice takes 0.2 to 0.8 % longer than the better way on
    // average; with the rates of 128 for heads of 64 it took 2.5 to 4.4 %.
    const double tile_bytes = 2.0 * kvt::mx_page_bytes(pool->head_dim) * kvt::kDecKeysPerTile / kvt::kBlock;
    const MxRates& r = mx_rates(pool->head_dim, rows > 16 && longest_message > 1);
    const double stream = (double)work * hkv * tile_bytes / r.stream;
    const int64_t first = cus * n / (hkv * chunks);   // sequences that have a CU of their own ...
    const int64_t start = std::max<int64_t>(1, 2 * cus * n / (hkv * chunks));   // ... and that start at once
    const double beside = n > start ? longest : n > first ? mx_tiles(seqs, p.order[c0 + first]) : 0;
    const double last = n > start ? mx_tiles(seqs, p.order[c0 + n - 1]) : 0;
    const double alone = std::max(r.tile * longest + r.beside * beside,
                                  stream * (n > first ? 1.0 : r.stream / r.one) + r.tile * last);
    if (alone <= r.join + std::max(r.tile * share, stream) + r.merge * n * share / total) share = total;
    bool split = false;
    int64_t begin = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t end = begin + mx_tiles(seqs, p.order[c0 + i]);
      const int parts = (int)((end - 1) / share - begin / share + 1);
      split = split || parts > 1;
      p.parts[c0 + i] = parts;
      if (parts > 1) p.part_rows += (int64_t)parts * seqs->suffix_len[p.order[c0 + i]] * num_q_heads;
      begin = end;
    }
    p.share.push_back(split ? (int32_t)share : 0);
  }
  if (p.part_rows > INT32_MAX) {
    p.parts.assign(B, 1);
    p.share.assign(p.share.size(), 0);
    p.part_rows = 0;
  }
  if (p.part_rows > 0) p.ws_bytes = mx_part_o_bytes(pool, p.part_rows) + (size_t)p.part_rows * 2 * sizeof(float);
  return p;
}

// Launches of a call of few rows: the shares, then the join of what they split.
kvt_status launch_mx_few(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads, float scale,
                         void* out, float* lse, int64_t T, void* workspace, size_t workspace_bytes, void* stream) {
  MxDecodePlan plan = mx_decode_plan(pool, seqs, num_q_heads);
  if (plan.ws_bytes > 0) {
    if (workspace == nullptr && workspace_bytes == 0) {   // no scratch offered: run unsplit
      plan.parts.assign(seqs->num_seqs, 1);
      plan.share.assign(plan.share.size(), 0);
      plan.ws_bytes = 0;
    } else {
      if (workspace == nullptr || workspace_bytes < plan.ws_bytes) return KVT_ERR_WORKSPACE;
      if (!aligned16(workspace) || !workspace_apart(pool, q, out, lse, num_q_heads, T, workspace, plan.ws_bytes))
        return KVT_ERR_INVALID_ARG;
    }
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  kvt::MxDecodeArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.out = out;
  a.lse = lse;
  a.block_table = seqs->block_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = pool->num_kv_heads;
  a.group = num_q_heads / pool->num_kv_heads;
  a.scale_log2 = scale * 1.4426950408889634f;
  if (plan.ws_bytes > 0) {
    a.part_o = reinterpret_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + mx_part_o_bytes(pool, plan.part_rows));
  }
  kvt::MxJoinArgs join;
  join.part_o = a.part_o;
  join.part_ml = a.part_ml;
  join.out = out;
  join.lse = lse;
  std::vector<int32_t> row_off(seqs->num_seqs + 1, 0);
  for (int b = 0; b < seqs->num_seqs; ++b) row_off[b + 1] = row_off[b] + seqs->suffix_len[b];
  int64_t part_row = 0;
  for (int c0 = 0, launch = 0; c0 < seqs->num_seqs; c0 += kvt::kSeqsPerLaunch, ++launch) {
    const int n = std::min(kvt::kSeqsPerLaunch, seqs->num_seqs - c0);
    a.nseq = n;
    a.share = plan.share[launch];
    a.chunks = plan.chunks[launch];
    join.nseq = 0;
    join.row_begin[0] = 0;
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) {
      const int b = plan.order[c0 + i], parts = plan.parts[c0 + i];
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row_off[b]};
      a.tile_begin[i] = (int32_t)tiles;
      a.part_row[i] = (int32_t)part_row;
      tiles += mx_tiles(seqs, b);
      if (parts > 1) {
        const int32_t rows = seqs->suffix_len[b] * num_q_heads;
        join.part_row[join.nseq] = (int32_t)part_row;
        join.row[join.nseq] = row_off[b] * num_q_heads;
        join.parts[join.nseq] = (uint8_t)parts;
        join.row_begin[join.nseq + 1] = join.row_begin[join.nseq] + rows;
        ++join.nseq;
        part_row += (int64_t)parts * rows;
      }
    }
    if (tiles > INT32_MAX / 2) return KVT_ERR_INVALID_ARG;   // (the kernel adds a share to a tile)
    a.tile_begin[n] = (int32_t)tiles;
    const int64_t slots = a.share > 0 ? (tiles + a.share - 1) / a.share : n;
    const int64_t grid = slots * pool->num_kv_heads * a.chunks;
    if (grid > INT32_MAX) return KVT_ERR_INVALID_ARG;
    hipError_t e = kvt::launch_mx_decode(a, pool->dtype, pool->head_dim, (int)grid, s);
    if (e == hipSuccess && join.nseq > 0) e = kvt::launch_mx_join(join, pool->dtype, pool->head_dim, s);
    if (e != hipSuccess) return device_error(e);
  }
  return KVT_OK;
}

// Token rows of a 4-bit append or read; fills the launch arguments.
kvt_status check_mx_rows(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_rows* k, const kvt_rows* v, bool writes,
                         int64_t* T, kvt::MxRowsArgs* a) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  if ((st = check_seqs(seqs, T)) != KVT_OK) return st;
  if (k == nullptr || v == nullptr) return KVT_ERR_INVALID_ARG;
  const int es = elem_bytes(pool->dtype);
  const int64_t width = (int64_t)pool->num_kv_heads * pool->head_dim;
  Rows kr, vr;
  if ((st = check_rows(k, *T, width, es, &kr)) != KVT_OK) return st;
  if ((st = check_rows(v, *T, width, es, &vr)) != KVT_OK) return st;
  const size_t held = pool_tensor_bytes(pool, true);
  for (const Rows* r : {&kr, &vr})
    for (const void* p : {(const void*)pool->k, (const void*)pool->v})
      if (overlaps((const void*)r->first, r->extent(), p, held)) return KVT_ERR_INVALID_ARG;
  if (writes ? rows_touch(kr, vr) : overlaps(pool->k, held, pool->v, held)) return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  a->k = k->data;
  a->v = v->data;
  a->k_stride = k->stride;
  a->v_stride = v->stride;
  a->k_pool = pool->k;
  a->v_pool = pool->v;
  a->block_table = seqs->block_table;
  a->num_blocks = pool->num_blocks;
  a->max_blocks = seqs->max_blocks;
  a->num_kv_heads = pool->num_kv_heads;
  return KVT_OK;
}

kvt_status launch_mx_rows(kvt::MxRowsArgs& a, const kvt_pool* pool, const kvt_seqs* seqs, bool writes, void* stream) {
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  int32_t row = 0;
  for (int b0 = 0; b0 < seqs->num_seqs; b0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, seqs->num_seqs - b0);
    a.nseq = n;
    a.row_begin = row;
    for (int i = 0; i < n; ++i) {
      const int b = b0 + i;
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row};
      row += seqs->suffix_len[b];
    }
    a.rows = row - a.row_begin;
    const hipError_t e = writes ? kvt::launch_mx_read(a, pool->dtype, pool->head_dim, s)
                                : kvt::launch_mx_append(a, pool->dtype, pool->head_dim, s);
    if (e != hipSuccess) return device_error(e);
  }
  return KVT_OK;
}

// Extent of rows [B][Hkv] of `used` values each, `stride` apart; 0: too large.
size_t head_rows_bytes(const kvt_pool* pool, int num_seqs, int64_t stride, int64_t used) {
  const int64_t rows = (int64_t)num_seqs * pool->num_kv_heads;
  if (stride > INT64_MAX / 8 / rows) return 0;
  return (size_t)((rows - 1) * stride + used) * 4;
}

int64_t longest_sequence(const kvt_seqs* seqs) {
  int64_t most = 0;
  for (int b = 0; b < seqs->num_seqs; ++b)
    most = std::max(most, (int64_t)seqs->prefix_len[b] + seqs->suffix_len[b]);
  return most;
}

kvt_status attention_weights(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                             float scale, const float* lse, float* weights, int64_t stride, int32_t scores,
                             void* stream, bool mx) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  if (scores != KVT_WEIGHTS_EXACT && scores != KVT_WEIGHTS_ROUNDED) return KVT_ERR_INVALID_ARG;
  int64_t T = 0;
  if ((st = check_seqs(seqs, &T)) != KVT_OK) return st;
  if (q == nullptr || lse == nullptr || weights == nullptr || !aligned16(q) || ((uintptr_t)lse & 3) != 0 ||
      ((uintptr_t)weights & 3) != 0)
    return KVT_ERR_INVALID_ARG;
  if (!heads_ok(pool, num_q_heads, T)) return KVT_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return KVT_ERR_INVALID_ARG;
  const int B = seqs->num_seqs, G = num_q_heads / pool->num_kv_heads;
  const int64_t most = longest_sequence(seqs);
  const size_t bytes = stride < most ? 0 : head_rows_bytes(pool, B, stride, most);
  if (bytes == 0) return KVT_ERR_INVALID_ARG;
  const size_t rows = (size_t)T * num_q_heads, held = pool_tensor_bytes(pool, mx);
  if (overlaps(weights, bytes, q, rows * pool->head_dim * elem_bytes(pool->dtype)) ||
      overlaps(weights, bytes, lse, rows * sizeof(float)) || overlaps(weights, bytes, pool->k, held) ||
      overlaps(weights, bytes, pool->v, held))
    return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;

  kvt::WeightsArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k_pool = pool->k;
  a.lse = lse;
  a.weights = weights;
  a.stride = stride;
  a.block_table = seqs->block_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = pool->num_kv_heads;
  a.group = G;
  // 2^(32 + s) / G rounded up, 2^s < G <= 2^(s + 1): at least 2^31, and off by less
  // than 1, so that x * by_group is off by less than x and the quotient is exact while
  // x * G < 2^(32 + s)
  while ((int64_t)2 << a.group_shift < G) ++a.group_shift;
  a.by_group = G == 1 ? 0u : (uint32_t)((((uint64_t)1 << (32 + a.group_shift)) + G - 1) / G);
  a.scale_log2 = scale * 1.4426950408889634f;
  const bool rounded = scores == KVT_WEIGHTS_ROUNDED && pool->dtype == KVT_DTYPE_F32;
  const int format = mx ? kvt::kMx : rounded ? kvt::kRounded : pool->dtype;
  const std::vector<int> order = longest_first(seqs);
  int64_t most_rows = 0;
  std::vector<int32_t> row_off(B + 1, 0);
  for (int b = 0; b < B; ++b) {
    row_off[b + 1] = row_off[b] + seqs->suffix_len[b];
    most_rows = std::max(most_rows, (int64_t)seqs->suffix_len[b] * G);
  }
  // up to the 32 rows that it takes, the step kernel streams the keys (8 new tokens,
  // 32/8 heads of 128, 16 contexts of 8000: 59.9 us, by the turn kernel 67.5; over
  // 4-bit pages 23.2 and 41.6; one of 32000 20.0 and 17.1)
  const bool step = most_rows <= 32;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  for (int c0 = 0; c0 < B; c0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, B - c0);
    a.nseq = n;
    int64_t units = 0, narrow = 0;
    const int keys = step ? kvt::kWeightsStepKeys : kvt::kWeightsWideKeys;
    // turn: the rows of every sequence are one stage, which stays in LDS while the
    // keys stream (32/8 heads of 128: 16 new tokens over 32000 keys 18.6 us, 28.8 a
    // tile at a time; 8 sequences adding 64 over 8000 each 53.3, 83.8)
    bool once = !step;
    for (int i = 0; i < n; ++i) {
      const int b = order[c0 + i];
      const int64_t len = (int64_t)seqs->prefix_len[b] + seqs->suffix_len[b];
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row_off[b]};
      units += (len + keys - 1) / keys;
      once = once && (int64_t)seqs->suffix_len[b] * G <= kvt::weights_stage_rows(pool->dtype);
    }
    // (the first sequence is the longest)
    const int64_t longest = ((int64_t)a.seq[0].prefix + a.seq[0].suffix + keys - 1) / keys;
    a.tiles = once ? (int32_t)std::min((units * pool->num_kv_heads + device_cus() - 1) / device_cus(), longest) : 0;
    // turn: wide workgroups in whole rounds of the CUs, and what a last, mostly
    // empty round would hold as narrow ones.  A narrow one has an eighth of the keys
    // but loads as many rows, and a round of them takes 0.4 of a wide one's time:
    // one round pays (32/8 heads of 128, 512 new tokens over 8192: 54.4 us, 78.8 with
    // wide ones only; fp32 192, 281), and two where the rows are many (512 over 9216:
    // 69.3, 78.8, fp32 229, 281; 140, 560 rows: 33.3, 32.5; 70: 26.4, 22.6).
    int64_t drop = 0;   // wide workgroups of each kv-head that become narrow ones
    if (!step && !once) {
      units = 0;
      int64_t rest = 0;   // narrow ones in any case
      for (int i = 0; i < n; ++i) {
        const int64_t len = (int64_t)a.seq[i].prefix + a.seq[i].suffix;
        units += len / keys;
        rest += (len % keys + 31) / 32;
      }
      const int64_t excess = units * pool->num_kv_heads % device_cus();
      const int64_t thin = (excess * 8 + rest * pool->num_kv_heads + device_cus() - 1) / device_cus();   // rounds of narrow ones
      const bool many = most_rows > (pool->dtype == KVT_DTYPE_BF16 ? 1024 : 768);
      if (thin < 2 || (thin == 2 && many)) drop = (excess + pool->num_kv_heads - 1) / pool->num_kv_heads;
    }
    units = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t len = (int64_t)a.seq[i].prefix + a.seq[i].suffix;
      a.unit_begin[i] = (int32_t)units;
      a.narrow_begin[i] = (int32_t)narrow;
      if (step) {
        units += (len + keys - 1) / keys;
      } else if (once) {
        units += ((len + keys - 1) / keys + a.tiles - 1) / a.tiles;
      } else {
        const int64_t wide = len / keys - std::min(len / keys, drop);
        drop -= len / keys - wide;
        units += wide;
        narrow += (len - wide * keys + 31) / 32;
      }
      if ((units + narrow) * pool->num_kv_heads > INT32_MAX / 2) return KVT_ERR_INVALID_ARG;
    }
    a.unit_begin[n] = (int32_t)units;
    a.narrow_begin[n] = (int32_t)narrow;
    hipError_t e;
    if (step) {
      // Loads of two or three workgroups keep a CU busy, more end at different times.
      // One context of 131000 and 48 of 1024..16384, 32/8 heads of 128, with 2, 3 and
      // 4 on a CU: bf16 54.6, 54.9, 60.1 us and 119.0, 121.3, 124.3; 4-bit 19.9,
      // 18.8, 20.0 and 40.0, 37.7, 38.6, with fp32 queries 22.2, 21.0, 21.8 (one);
      // fp32 103, 106, 109
      const int64_t slots = std::max<int64_t>(1, (mx ? 3 : 2) * (int64_t)device_cus() / pool->num_kv_heads);
      a.share = (int32_t)std::max<int64_t>(4, (units + slots - 1) / slots);
      e = kvt::launch_weights_step(a, format, pool->dtype, pool->head_dim,
                                   (int)((units + a.share - 1) / a.share) * pool->num_kv_heads, s);
    } else {
      e = kvt::launch_weights_turn(a, format, pool->dtype, pool->head_dim, (int)(units + narrow) * pool->num_kv_heads,
                                   s);
    }
    if (e != hipSuccess) return device_error(e);
  }
  return KVT_OK;
}

kvt_status evict(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_eviction* ev, void* stream, bool mx) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  int64_t T = 0;
  if ((st = check_seqs(seqs, &T)) != KVT_OK) return st;
  if (ev == nullptr || ev->keep == nullptr || ev->weights == nullptr || ev->to_table == nullptr ||
      ev->positions == nullptr || ev->sinks < 0 || ev->recent < 0 || ev->to_max_blocks < 1)
    return KVT_ERR_INVALID_ARG;
  for (const void* p : {(const void*)ev->weights, (const void*)ev->positions, (const void*)ev->weights_out})
    if (((uintptr_t)p & 3) != 0) return KVT_ERR_INVALID_ARG;
  const int B = seqs->num_seqs;
  std::vector<int32_t> kept(B);
  int64_t most_kept = 0;
  for (int b = 0; b < B; ++b) {
    const int64_t L = (int64_t)seqs->prefix_len[b] + seqs->suffix_len[b];
    if (ev->keep[b] < 1) return KVT_ERR_INVALID_ARG;
    if (L > ev->keep[b] && (int64_t)ev->sinks + ev->recent > ev->keep[b]) return KVT_ERR_INVALID_ARG;
    kept[b] = (int32_t)std::min<int64_t>(L, ev->keep[b]);
    if ((kept[b] + kvt::kBlock - 1) / kvt::kBlock > ev->to_max_blocks) return KVT_ERR_INVALID_ARG;
    most_kept = std::max<int64_t>(most_kept, kept[b]);
  }
  const int64_t most = longest_sequence(seqs);
  const size_t in_bytes = ev->weights_stride < most ? 0 : head_rows_bytes(pool, B, ev->weights_stride, most);
  const size_t out_bytes =
      ev->out_stride < most_kept || ev->out_stride > INT32_MAX ? 0 : head_rows_bytes(pool, B, ev->out_stride, ev->out_stride);
  if (in_bytes == 0 || out_bytes == 0) return KVT_ERR_INVALID_ARG;
  const size_t held = pool_tensor_bytes(pool, mx);
  auto in_pool = [&](const void* p, size_t n) { return overlaps(p, n, pool->k, held) || overlaps(p, n, pool->v, held); };
  if (overlaps(ev->positions, out_bytes, ev->weights, in_bytes) || in_pool(ev->positions, out_bytes) ||
      in_pool(ev->weights, in_bytes) || overlaps(pool->k, held, pool->v, held))
    return KVT_ERR_INVALID_ARG;
  if (ev->weights_out != nullptr &&
      (overlaps(ev->weights_out, out_bytes, ev->weights, in_bytes) ||
       overlaps(ev->weights_out, out_bytes, ev->positions, out_bytes) || in_pool(ev->weights_out, out_bytes)))
    return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  if (ev->to_table_host != nullptr) {
    // targets: inside the pool, each page once, and none that the call reads
    std::unordered_set<int32_t> seen;
    for (int b = 0; b < B; ++b)
      for (int i = 0; i < (kept[b] + kvt::kBlock - 1) / kvt::kBlock; ++i) {
        const int32_t id = ev->to_table_host[(int64_t)b * ev->to_max_blocks + i];
        if (id < 0 || id >= pool->num_blocks || !seen.insert(id).second) return KVT_ERR_OUT_OF_RANGE;
      }
    for (int b = 0; b < B && seqs->block_table_host != nullptr; ++b) {
      const int64_t L = (int64_t)seqs->prefix_len[b] + seqs->suffix_len[b];
      for (int64_t i = 0; i < (L + kvt::kBlock - 1) / kvt::kBlock; ++i)
        if (seen.count(seqs->block_table_host[(int64_t)b * seqs->max_blocks + i])) return KVT_ERR_OUT_OF_RANGE;
    }
  }

  const std::vector<int> order = longest_first(seqs);
  for (int c0 = 0; c0 < B; c0 += kvt::kSeqsPerLaunch) {   // every launch, before the first one
    int64_t pages = 0;
    for (int i = c0; i < std::min(B, c0 + kvt::kSeqsPerLaunch); ++i)
      pages += (kept[order[i]] + kvt::kBlock - 1) / kvt::kBlock;
    if (pages * pool->num_kv_heads > INT32_MAX) return KVT_ERR_INVALID_ARG;
  }

  kvt::EvictArgs a;
  std::memset(&a, 0, sizeof(a));
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.weights = ev->weights;
  a.stride = ev->weights_stride;
  a.positions = ev->positions;
  a.weights_out = ev->weights_out;
  a.out_stride = ev->out_stride;
  a.block_table = seqs->block_table;
  a.to_table = ev->to_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.to_max_blocks = ev->to_max_blocks;
  a.num_kv_heads = pool->num_kv_heads;
  a.sinks = ev->sinks;
  a.recent = ev->recent;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  for (int c0 = 0; c0 < B; c0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, B - c0);
    int64_t pages = 0;
    a.nseq = n;
    for (int i = 0; i < n; ++i) {
      const int b = order[c0 + i];
      a.seq[i] = kvt::EvictDesc{b, seqs->prefix_len[b] + seqs->suffix_len[b], kept[b]};
      a.unit_begin[i] = (int32_t)pages;
      pages += (kept[b] + kvt::kBlock - 1) / kvt::kBlock;
    }
    a.unit_begin[n] = (int32_t)pages;
    hipError_t e = kvt::launch_evict_select(a, s);
    if (e != hipSuccess) return device_error(e);
    constexpr int32_t kMost = 1 << 23;   // a launch holds less than 2^32 threads
    const int32_t blocks = (int32_t)(pages * pool->num_kv_heads);
    for (a.first_block = 0; a.first_block < blocks; a.first_block += std::min(kMost, blocks - a.first_block)) {
      e = kvt::launch_evict_move(a, mx ? kvt::kMx : pool->dtype, pool->head_dim, std::min(kMost, blocks - a.first_block), s);
      if (e != hipSuccess) return device_error(e);
    }
  }
  return KVT_OK;
}

// Pages to or from pinned host memory; `mx`: 4-bit pages.
kvt_status copy_blocks(const kvt_pool* pool, const int32_t* block_ids, const int32_t* block_ids_host, int64_t num_ids,
                       void* host, int32_t direction, void* stream, bool mx) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  if (num_ids < 0 || (num_ids > 0 && (block_ids == nullptr || host == nullptr))) return KVT_ERR_INVALID_ARG;
  if (direction != KVT_COPY_TO_HOST && direction != KVT_COPY_TO_DEVICE) return KVT_ERR_INVALID_ARG;
  if (num_ids == 0) return KVT_OK;
  if (mx && !aligned16(host)) return KVT_ERR_INVALID_ARG;   // (bytes can begin anywhere)
  const int64_t page_bytes = (int64_t)pool->num_kv_heads * page_bytes_of_head(pool, mx);
  if (num_ids > (INT64_MAX / 4) / (2 * page_bytes)) return KVT_ERR_INVALID_ARG;
  if (block_ids_host != nullptr) {
    std::unordered_set<int32_t> seen;
    for (int64_t i = 0; i < num_ids; ++i) {
      const int32_t id = block_ids_host[i];
      if (id < 0 || id >= pool->num_blocks) return KVT_ERR_OUT_OF_RANGE;
      // two host pages landing on one pool page would race
      if (direction == KVT_COPY_TO_DEVICE && !seen.insert(id).second) return KVT_ERR_OUT_OF_RANGE;
    }
  }
  // the host side must be pinned memory the device can address
  hipPointerAttribute_t attr;
  std::memset(&attr, 0, sizeof(attr));
  if (hipPointerGetAttributes(&attr, host) != hipSuccess) {
    (void)hipGetLastError();
    return KVT_ERR_INVALID_ARG;
  }
  if (attr.type != hipMemoryTypeHost) return KVT_ERR_INVALID_ARG;
  void* host_dev = attr.devicePointer != nullptr ? attr.devicePointer : host;

  kvt::CopyArgs a;
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.ids = block_ids;
  a.n = num_ids;
  a.host = host_dev;
  a.page_bytes = page_bytes;
  a.num_blocks = pool->num_blocks;
  a.to_host = direction == KVT_COPY_TO_HOST ? 1 : 0;
  const int64_t pieces = num_ids * 2 * page_bytes / 16;
  const int grid = (int)std::min<int64_t>((pieces + 255) / 256, 8192);
  const hipError_t e = kvt::launch_copy_blocks(a, grid, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? KVT_OK : device_error(e);
}

}  // namespace

extern "C" {

const char* kvt_status_str(kvt_status s) {
  switch (s) {
    case KVT_OK: return "ok";
    case KVT_ERR_INVALID_ARG: return "invalid argument";
    case KVT_ERR_UNSUPPORTED: return "unsupported shape or dtype";
    case KVT_ERR_OUT_OF_RANGE: return "block id out of range or duplicate append target";
    case KVT_ERR_WORKSPACE: return "workspace too small";
    case KVT_ERR_DEVICE: return "HIP launch failed";
    case KVT_ERR_SCRATCH_LIMIT: return "split partials exceed the static scratch (KVT_NOALLOC_SCRATCH_BYTES)";
  }
  return "unknown status";
}

int kvt_last_hip_error(void) { return g_last_hip_error; }

kvt_status kvt_append_kv(const kvt_pool* pool, const kvt_seqs* seqs, const void* k_new, const void* v_new,
                         void* stream) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  int64_t T = 0;
  if ((st = check_seqs(seqs, &T)) != KVT_OK) return st;
  if (k_new == nullptr || v_new == nullptr || !aligned16(k_new) || !aligned16(v_new)) return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  const size_t pool_bytes = (size_t)pool->num_blocks * pool->num_kv_heads * kvt::kBlock * pool->head_dim *
                            elem_bytes(pool->dtype);
  const size_t new_bytes = (size_t)T * pool->num_kv_heads * pool->head_dim * elem_bytes(pool->dtype);
  for (const void* src : {k_new, v_new})
    for (const void* dst : {(const void*)pool->k, (const void*)pool->v})
      if (overlaps(src, new_bytes, dst, pool_bytes)) return KVT_ERR_INVALID_ARG;
  if ((st = check_append_targets(seqs, T)) != KVT_OK) return st;

  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  kvt::AppendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.k_new = k_new;
  a.v_new = v_new;
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.block_table = seqs->block_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.num_kv_heads = pool->num_kv_heads;
  int32_t row = 0;
  for (int b0 = 0; b0 < seqs->num_seqs; b0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, seqs->num_seqs - b0);
    a.nseq = n;
    a.row_begin = row;
    for (int i = 0; i < n; ++i) {
      const int b = b0 + i;
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row};
      row += seqs->suffix_len[b];
    }
    a.rows = row - a.row_begin;
    const hipError_t e = kvt::launch_append(a, pool->dtype, pool->head_dim, s);
    if (e != hipSuccess) return device_error(e);
  }
  return KVT_OK;
}

kvt_status kvt_rotate(const kvt_rotary* rotary, const kvt_rows* x, int64_t num_tokens, int32_t num_heads,
                      int32_t head_dim, int32_t dtype, const kvt_rows* out, void* stream) {
  if (head_dim != 64 && head_dim != 128) return KVT_ERR_UNSUPPORTED;
  if (dtype != KVT_DTYPE_BF16 && dtype != KVT_DTYPE_F32) return KVT_ERR_UNSUPPORTED;
  kvt::RotaryArgs a;
  std::memset(&a, 0, sizeof(a));
  kvt_status st = check_rotary(rotary, head_dim, &a);
  if (st != KVT_OK) return st;
  if (x == nullptr || out == nullptr || num_tokens < 0 || num_heads < 1) return KVT_ERR_INVALID_ARG;
  if (num_tokens == 0) return KVT_OK;
  if (num_tokens > INT32_MAX / num_heads || rotary->positions == nullptr) return KVT_ERR_INVALID_ARG;
  const int64_t width = (int64_t)num_heads * head_dim;
  Rows from, to;
  if ((st = check_rows(x, num_tokens, width, elem_bytes(dtype), &from)) != KVT_OK) return st;
  if ((st = check_rows(out, num_tokens, width, elem_bytes(dtype), &to)) != KVT_OK) return st;
  if (!rows_same(from, to) && rows_touch(from, to)) return KVT_ERR_INVALID_ARG;
  if (covers_positions(to, rotary)) return KVT_ERR_INVALID_ARG;
  a.q = x->data;
  a.q_out = out->data;
  a.q_stride = x->stride;
  a.q_out_stride = out->stride;
  a.num_q_heads = num_heads;
  a.rows = a.total_rows = num_tokens;
  const hipError_t e = kvt::launch_rotary(a, dtype, head_dim, device_cus(), reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? KVT_OK : device_error(e);
}

kvt_status kvt_append_kv_rotary(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_rotary* rotary,
                                const kvt_rows* k_new, const kvt_rows* v_new, const kvt_rows* q, int32_t num_q_heads,
                                const kvt_rows* q_out, void* stream) try {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  int64_t T = 0;
  if ((st = check_seqs(seqs, &T)) != KVT_OK) return st;
  kvt::RotaryArgs a;
  std::memset(&a, 0, sizeof(a));
  if ((st = check_rotary(rotary, pool->head_dim, &a)) != KVT_OK) return st;
  if (rotary->positions == nullptr && rotary->num_axes != 1) return KVT_ERR_INVALID_ARG;
  if (k_new == nullptr || v_new == nullptr || (q == nullptr) != (q_out == nullptr)) return KVT_ERR_INVALID_ARG;
  if (q == nullptr ? num_q_heads != 0 : !heads_ok(pool, num_q_heads, T)) return KVT_ERR_INVALID_ARG;
  const int es = elem_bytes(pool->dtype);
  const int64_t kv_width = (int64_t)pool->num_kv_heads * pool->head_dim;
  Rows k, v, qi, qo;
  if ((st = check_rows(k_new, T, kv_width, es, &k)) != KVT_OK) return st;
  if ((st = check_rows(v_new, T, kv_width, es, &v)) != KVT_OK) return st;
  const size_t pool_bytes = (size_t)pool->num_blocks * kvt::kBlock * kv_width * es;
  auto in_pool = [&](const Rows& r) {
    return overlaps((const void*)r.first, r.extent(), pool->k, pool_bytes) ||
           overlaps((const void*)r.first, r.extent(), pool->v, pool_bytes);
  };
  if (in_pool(k) || in_pool(v)) return KVT_ERR_INVALID_ARG;
  if (q != nullptr) {
    const int64_t q_width = (int64_t)num_q_heads * pool->head_dim;
    if ((st = check_rows(q, T, q_width, es, &qi)) != KVT_OK) return st;
    if ((st = check_rows(q_out, T, q_width, es, &qo)) != KVT_OK) return st;
    if (in_pool(qi) || in_pool(qo) || rows_touch(qo, k) || rows_touch(qo, v)) return KVT_ERR_INVALID_ARG;
    if (!rows_same(qi, qo) && rows_touch(qi, qo)) return KVT_ERR_INVALID_ARG;
    if (covers_positions(qo, rotary)) return KVT_ERR_INVALID_ARG;
    a.q = q->data;
    a.q_out = q_out->data;
    a.q_stride = q->stride;
    a.q_out_stride = q_out->stride;
    a.num_q_heads = num_q_heads;
  }
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  if ((st = check_append_targets(seqs, T)) != KVT_OK) return st;

  a.k_new = k_new->data;
  a.v_new = v_new->data;
  a.k_stride = k_new->stride;
  a.v_stride = v_new->stride;
  a.k_pool = pool->k;
  a.v_pool = pool->v;
  a.block_table = seqs->block_table;
  a.num_blocks = pool->num_blocks;
  a.max_blocks = seqs->max_blocks;
  a.num_kv_heads = pool->num_kv_heads;
  a.total_rows = T;
  int32_t row = 0;
  for (int b0 = 0; b0 < seqs->num_seqs; b0 += kvt::kSeqsPerLaunch) {
    const int n = std::min(kvt::kSeqsPerLaunch, seqs->num_seqs - b0);
    a.nseq = n;
    a.row_begin = row;
    for (int i = 0; i < n; ++i) {
      const int b = b0 + i;
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row};
      row += seqs->suffix_len[b];
    }
    a.rows = row - a.row_begin;
    const hipError_t e =
        kvt::launch_rotary(a, pool->dtype, pool->head_dim, device_cus(), reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) return device_error(e);
  }
  return KVT_OK;
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

size_t kvt_extend_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK) return 0;
  if (!heads_ok(pool, num_q_heads, T)) return 0;
  return extend_plan(pool, seqs, num_q_heads, T).ws_bytes;
}

kvt_status kvt_extend_attention(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
  int64_t T = 0;
  const kvt_status st = check_extend(pool, seqs, q, num_q_heads, scale, out, lse, &T);
  if (st != KVT_OK) return st;
  ExtendPlan plan = extend_plan(pool, seqs, num_q_heads, T);
  const kvt_status fit = fit_workspace(&plan, pool, T * num_q_heads, workspace, workspace_bytes);
  if (fit != KVT_OK) return fit;
  return launch_extend_plan(pool, seqs, q, num_q_heads, scale, out, lse, T, plan, workspace, stream);
}

kvt_status kvt_extend_attention_noalloc(const kvt_pool* pool, const kvt_seqs* seqs, const void* q,
                                        int32_t num_q_heads, float scale, void* out, float* lse, void* stream) {
  int64_t T = 0;
  const kvt_status st = check_extend(pool, seqs, q, num_q_heads, scale, out, lse, &T);
  if (st != KVT_OK) return st;
  // the same plan as kvt_extend_attention with a large enough workspace, so
  // both give the same bits, partials in the static scratch; but a call that
  // splits only to fill the chip (its base count is 1) stays unsplit and off
  // the scratch, so that it may overlap other calls on other streams
  ExtendPlan plan = extend_plan(pool, seqs, num_q_heads, T);
  if (plan.nsplit_base == 1) plan.nsplit = 1, plan.heaviest = 0.0;
  void* ws = nullptr;
  if (plan.nsplit > 1) {
    if (plan.ws_bytes > (size_t)KVT_NOALLOC_SCRATCH_BYTES) return KVT_ERR_SCRATCH_LIMIT;
    const hipError_t e = kvt::noalloc_scratch(&ws);
    if (e != hipSuccess) return device_error(e);
  }
  return launch_extend_plan(pool, seqs, q, num_q_heads, scale, out, lse, T, plan, ws, stream);
}

kvt_status kvt_copy_blocks(const kvt_pool* pool, const int32_t* block_ids, const int32_t* block_ids_host,
                           int64_t num_ids, void* host, int32_t direction, void* stream) try {
  return copy_blocks(pool, block_ids, block_ids_host, num_ids, host, direction, stream, false);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

size_t kvt_cascade_workspace_bytes_ex(const kvt_pool* pool, const kvt_seqs* seqs, int32_t shared_len,
                                      int32_t mode, int32_t num_q_heads) {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK) return 0;
  if (!heads_ok(pool, num_q_heads, T)) return 0;
  if (check_shared(seqs, shared_len) != KVT_OK || !mode_ok(mode)) return 0;
  return cascade_plan(pool, seqs, shared_len, num_q_heads, T, mode).ws_bytes;
}

size_t kvt_cascade_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t shared_len,
                                   int32_t num_q_heads) {
  return kvt_cascade_workspace_bytes_ex(pool, seqs, shared_len, KVT_CASCADE_AUTO, num_q_heads);
}

int32_t kvt_cascade_uses_shared_pass(const kvt_pool* pool, const kvt_seqs* seqs, int32_t shared_len,
                                     int32_t num_q_heads) {
  if (check_pool(pool) != KVT_OK) return -1;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK) return -1;
  if (!heads_ok(pool, num_q_heads, T)) return -1;
  if (check_shared(seqs, shared_len) != KVT_OK) return -1;
  return cascade_plan(pool, seqs, shared_len, num_q_heads, T, KVT_CASCADE_AUTO, true).use_shared ? 1 : 0;
}

kvt_status kvt_cascade_extend_attention(const kvt_pool* pool, const kvt_seqs* seqs, int32_t shared_len,
                                        const void* q, int32_t num_q_heads, float scale, void* out, float* lse,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  return kvt_cascade_extend_attention_ex(pool, seqs, shared_len, KVT_CASCADE_AUTO, q, num_q_heads, scale, out, lse,
                                         workspace, workspace_bytes, stream);
}

kvt_status kvt_cascade_extend_attention_ex(const kvt_pool* pool, const kvt_seqs* seqs, int32_t shared_len,
                                           int32_t mode, const void* q, int32_t num_q_heads, float scale, void* out,
                                           float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  int64_t T = 0;
  if ((st = check_seqs(seqs, &T)) != KVT_OK) return st;
  if ((st = check_shared(seqs, shared_len)) != KVT_OK) return st;
  if (!mode_ok(mode)) return KVT_ERR_INVALID_ARG;
  if (workspace == nullptr && workspace_bytes == 0)   // no scratch: the plain extend computes the same
    return kvt_extend_attention(pool, seqs, q, num_q_heads, scale, out, lse, nullptr, 0, stream);
  if (q == nullptr || out == nullptr) return KVT_ERR_INVALID_ARG;
  if (!heads_ok(pool, num_q_heads, T)) return KVT_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  if ((st = check_outputs(pool, q, num_q_heads, out, lse, T)) != KVT_OK) return st;
  ExtendPlan plan = cascade_plan(pool, seqs, shared_len, num_q_heads, T, mode);
  if (workspace == nullptr) return KVT_ERR_WORKSPACE;
  if (!plan.use_shared) {
    if ((st = fit_workspace(&plan, pool, T * num_q_heads, workspace, workspace_bytes)) != KVT_OK) return st;
  } else if (workspace_bytes < plan.ws_bytes) {   // room for the base split counts?
    plan = cascade_plan(pool, seqs, shared_len, num_q_heads, T, mode, true);
    if (workspace_bytes < plan.ws_bytes) return KVT_ERR_WORKSPACE;
  }
  if (!aligned16(workspace)) return KVT_ERR_INVALID_ARG;
  if (!plan.use_shared)   // the plain extend is estimated faster: same result, same bits as kvt_extend_attention
    return launch_extend_plan(pool, seqs, q, num_q_heads, scale, out, lse, T, plan, workspace, stream);

  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int G = num_q_heads / pool->num_kv_heads;
  const int nparts = plan.nsplit_shared + plan.nsplit;
  ExtendPlan parts = plan;
  parts.nsplit = nparts;                       // partial buffers: the shared part's splits, then the private ones
  kvt::ExtendArgs a = base_args(pool, seqs, q, num_q_heads, scale, out, lse, T, parts, workspace);
  a.direct = 0;

  // One launch for both parts, the shared part's (longer) units first, so
  // the private parts' units fill the CUs the shared part leaves idle at
  // its end.  Shared part (sequence 0 of the first launch): every new token
  // of the batch against keys [0, shared_len), all of them visible (one
  // virtual sequence whose causal limits start at shared_len - 1), read
  // through the first sequence's table row, with its own key splits.
  // Private parts (the second group): each sequence over keys
  // [shared_len, P_b + i], causal.  Sequences beyond one launch's
  // descriptors go to further launches of private parts only.
  a.nsplit = plan.nsplit_shared;
  a.part_base = 0;
  a.kbeg = 0;
  a.kend = shared_len;
  a.kbeg2 = shared_len;
  a.kend2 = INT32_MAX;
  a.nsplit2 = plan.nsplit;
  a.part_base2 = plan.nsplit_shared;
  std::vector<int32_t> row_off(seqs->num_seqs + 1, 0);
  for (int b = 0; b < seqs->num_seqs; ++b) row_off[b + 1] = row_off[b] + seqs->suffix_len[b];
  size_t c0 = 0;
  for (bool first = true; first || c0 < plan.order.size(); first = false) {
    int n = 0;
    int32_t units = 0;
    if (first) {
      a.seq[0] = kvt::SeqDesc{plan.order[0], shared_len - 1, (int32_t)T, 0};
      a.last[0] = (uint8_t)plan.nsplit_shared;
      a.unit_begin[0] = 0;
      units = row_tiles((int32_t)T, G) * plan.nsplit_shared;
      n = 1;
    }
    a.second = first ? 1 : 0;
    for (; n < kvt::kSeqsPerLaunch && c0 < plan.order.size(); ++n, ++c0) {
      const int b = plan.order[c0];
      a.seq[n] = kvt::SeqDesc{b, seqs->prefix_len[b], seqs->suffix_len[b], row_off[b]};
      a.last[n] = (uint8_t)plan.nsplit;
      a.unit_begin[n] = units;
      units += row_tiles(seqs->suffix_len[b], G) * plan.nsplit;
    }
    a.nseq = n;
    a.unit_begin[n] = units;
    const int64_t grid = (int64_t)units * pool->num_kv_heads;
    if (grid > INT32_MAX) return KVT_ERR_INVALID_ARG;
    const hipError_t e = kvt::launch_extend(a, pool->dtype, pool->head_dim, (int)grid, s);
    if (e != hipSuccess) return device_error(e);
  }
  return combine(a, pool, out, lse, T, num_q_heads, nparts, false, s);
}

size_t kvt_decode_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK || T != seqs->num_seqs) return 0;
  if (!heads_ok(pool, num_q_heads, T)) return 0;
  if (num_q_heads / pool->num_kv_heads > kvt::kDecMaxGroup) return 0;
  return make_decode_plan(pool, seqs, num_q_heads).ws_bytes;
}

kvt_status kvt_decode_attention(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
  kvt_status st = check_pool(pool);
  if (st != KVT_OK) return st;
  int64_t T = 0;
  if ((st = check_seqs(seqs, &T)) != KVT_OK) return st;
  if (T != seqs->num_seqs) return KVT_ERR_INVALID_ARG;   // one new token per sequence
  if (q == nullptr || out == nullptr) return KVT_ERR_INVALID_ARG;
  if (!heads_ok(pool, num_q_heads, T)) return KVT_ERR_INVALID_ARG;
  if (num_q_heads / pool->num_kv_heads > kvt::kDecMaxGroup) return KVT_ERR_UNSUPPORTED;
  if (!(scale > 0.f) || !std::isfinite(scale)) return KVT_ERR_INVALID_ARG;
  if ((st = check_table_ids(pool, seqs)) != KVT_OK) return st;
  if ((st = check_outputs(pool, q, num_q_heads, out, lse, T)) != KVT_OK) return st;

  ExtendPlan plan = make_decode_plan(pool, seqs, num_q_heads);
  if ((st = fit_workspace(&plan, pool, T * num_q_heads, workspace, workspace_bytes)) != KVT_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int per_cu = decode_per_cu(pool, seqs, plan);
  kvt::ExtendArgs a = base_args(pool, seqs, q, num_q_heads, scale, out, lse, T, plan, workspace);
  for (size_t c0 = 0; c0 < plan.order.size(); c0 += kvt::kSeqsPerLaunch) {
    const int n = (int)std::min<size_t>(kvt::kSeqsPerLaunch, plan.order.size() - c0);
    a.nseq = n;
    for (int i = 0; i < n; ++i) {
      const int b = plan.order[c0 + i];
      a.seq[i] = kvt::SeqDesc{b, seqs->prefix_len[b], 1, b};   // row of sequence b is b
      a.unit_begin[i] = i * plan.nsplit;
    }
    a.unit_begin[n] = n * plan.nsplit;
    const int64_t grid = (int64_t)n * plan.nsplit * pool->num_kv_heads;
    const hipError_t e = kvt::launch_decode(a, pool->dtype, pool->head_dim, (int)grid, per_cu, s);
    if (e != hipSuccess) return device_error(e);
  }
  return plan.nsplit > 1 ? combine(a, pool, out, lse, T, num_q_heads, plan.nsplit, false, s) : KVT_OK;
}

size_t kvt_diff_extend_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) try {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK || !heads_ok(pool, num_q_heads, T)) return 0;
  return diff_extend_plan(pool, seqs, num_q_heads).ws_bytes;
} catch (const std::bad_alloc&) {
  return 0;
}

kvt_status kvt_diff_extend_attention(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                     float scale, const kvt_diff* diff, void* out, void* workspace,
                                     size_t workspace_bytes, void* stream) try {
  int64_t T = 0;
  const kvt_status st = check_diff(pool, seqs, q, num_q_heads, scale, diff, out, &T);
  if (st != KVT_OK) return st;
  DiffPlan plan = diff_extend_plan(pool, seqs, num_q_heads);
  return launch_diff(pool, seqs, q, num_q_heads, scale, diff, out, T, plan, false, workspace, workspace_bytes, stream);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

size_t kvt_diff_decode_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) try {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK || T != seqs->num_seqs || !heads_ok(pool, num_q_heads, T)) return 0;
  return diff_decode_plan(pool, seqs, num_q_heads).ws_bytes;
} catch (const std::bad_alloc&) {
  return 0;
}

kvt_status kvt_diff_decode_attention(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                     float scale, const kvt_diff* diff, void* out, void* workspace,
                                     size_t workspace_bytes, void* stream) try {
  int64_t T = 0;
  const kvt_status st = check_diff(pool, seqs, q, num_q_heads, scale, diff, out, &T);
  if (st != KVT_OK) return st;
  if (T != seqs->num_seqs) return KVT_ERR_INVALID_ARG;   // one new token per sequence
  DiffPlan plan = diff_decode_plan(pool, seqs, num_q_heads);
  return launch_diff(pool, seqs, q, num_q_heads, scale, diff, out, T, plan, true, workspace, workspace_bytes, stream);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_mx_append_kv(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_rows* k_new, const kvt_rows* v_new,
                            void* stream) try {
  kvt::MxRowsArgs a;
  std::memset(&a, 0, sizeof(a));
  int64_t T = 0;
  kvt_status st = check_mx_rows(pool, seqs, k_new, v_new, false, &T, &a);
  if (st != KVT_OK) return st;
  if ((st = check_append_targets(seqs, T)) != KVT_OK) return st;
  return launch_mx_rows(a, pool, seqs, false, stream);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_mx_read_kv(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_rows* k_out, const kvt_rows* v_out,
                          void* stream) try {
  kvt::MxRowsArgs a;
  std::memset(&a, 0, sizeof(a));
  int64_t T = 0;
  const kvt_status st = check_mx_rows(pool, seqs, k_out, v_out, true, &T, &a);
  if (st != KVT_OK) return st;
  return launch_mx_rows(a, pool, seqs, true, stream);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

size_t kvt_mx_extend_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) try {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK || !heads_ok(pool, num_q_heads, T)) return 0;
  if (mx_few_rows(pool, seqs, num_q_heads)) return mx_decode_plan(pool, seqs, num_q_heads).ws_bytes;
  return extend_plan(pool, seqs, num_q_heads, T).ws_bytes;
} catch (const std::bad_alloc&) {
  return 0;
}

kvt_status kvt_mx_extend_attention(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                   float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                   void* stream) try {
  int64_t T = 0;
  const kvt_status st = check_extend(pool, seqs, q, num_q_heads, scale, out, lse, &T, true);
  if (st != KVT_OK) return st;
  if (mx_few_rows(pool, seqs, num_q_heads))
    return launch_mx_few(pool, seqs, q, num_q_heads, scale, out, lse, T, workspace, workspace_bytes, stream);
  ExtendPlan plan = extend_plan(pool, seqs, num_q_heads, T);
  const kvt_status fit = fit_workspace(&plan, pool, T * num_q_heads, workspace, workspace_bytes);
  if (fit != KVT_OK) return fit;
  if (plan.nsplit > 1 && !workspace_apart(pool, q, out, lse, num_q_heads, T, workspace, plan.ws_bytes))
    return KVT_ERR_INVALID_ARG;
  return launch_extend_plan(pool, seqs, q, num_q_heads, scale, out, lse, T, plan, workspace, stream, true);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

size_t kvt_mx_decode_workspace_bytes(const kvt_pool* pool, const kvt_seqs* seqs, int32_t num_q_heads) try {
  if (check_pool(pool) != KVT_OK) return 0;
  int64_t T = 0;
  if (check_seqs(seqs, &T) != KVT_OK || T != seqs->num_seqs || !heads_ok(pool, num_q_heads, T)) return 0;
  return mx_decode_plan(pool, seqs, num_q_heads).ws_bytes;
} catch (const std::bad_alloc&) {
  return 0;
}

kvt_status kvt_mx_decode_attention(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                   float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                   void* stream) try {
  int64_t T = 0;
  const kvt_status st = check_extend(pool, seqs, q, num_q_heads, scale, out, lse, &T, true);
  if (st != KVT_OK) return st;
  if (T != seqs->num_seqs) return KVT_ERR_INVALID_ARG;   // one new token per sequence
  return launch_mx_few(pool, seqs, q, num_q_heads, scale, out, lse, T, workspace, workspace_bytes, stream);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_attention_weights(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                 float scale, const float* lse, float* weights, int64_t weights_stride,
                                 void* stream) try {
  return attention_weights(pool, seqs, q, num_q_heads, scale, lse, weights, weights_stride, KVT_WEIGHTS_EXACT, stream,
                           false);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_attention_weights_ex(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                    float scale, const float* lse, float* weights, int64_t weights_stride,
                                    int32_t scores, void* stream) try {
  return attention_weights(pool, seqs, q, num_q_heads, scale, lse, weights, weights_stride, scores, stream, false);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_mx_attention_weights(const kvt_pool* pool, const kvt_seqs* seqs, const void* q, int32_t num_q_heads,
                                    float scale, const float* lse, float* weights, int64_t weights_stride,
                                    void* stream) try {
  return attention_weights(pool, seqs, q, num_q_heads, scale, lse, weights, weights_stride, KVT_WEIGHTS_EXACT, stream,
                           true);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_evict(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_eviction* eviction, void* stream) try {
  return evict(pool, seqs, eviction, stream, false);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_mx_copy_blocks(const kvt_pool* pool, const int32_t* block_ids, const int32_t* block_ids_host,
                              int64_t num_ids, void* host, int32_t direction, void* stream) try {
  return copy_blocks(pool, block_ids, block_ids_host, num_ids, host, direction, stream, true);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

kvt_status kvt_mx_evict(const kvt_pool* pool, const kvt_seqs* seqs, const kvt_eviction* eviction, void* stream) try {
  return evict(pool, seqs, eviction, stream, true);
} catch (const std::bad_alloc&) {
  return device_error(hipErrorOutOfMemory);
}

}  // extern "C"
