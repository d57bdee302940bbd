// Eviction by accumulated weight, gfx950.
//
// Per sequence and kv-head, of L positions n = min(L, keep) stay: the first
// `sinks`, the last `recent`, and of those between them the heaviest, of equal
// ones the lowest positions.  Two launches:
//   * select: one workgroup per (sequence, kv-head).  The weights become 32-bit
//     keys in the same order.  The k-th largest is found 11, 11 and 10 bits at a
//     time from the top: a histogram of the keys that agree so far (integer
//     counts in LDS, so their order does not matter), then the bin that holds the
//     k-th.  Every wave owns a sixteenth of the positions, in order, so that its
//     ballots count what stays before a position, and the waves' totals the rest.
//     Bound by its instructions for each position: of 61083 positions the first
//     pass takes 8.8 us, the second 10.4, the last 7.5, the three counts 1.2 each;
//   * move: the kept rows into the other pages, 16 bytes a lane in the order of
//     the targets; reads are whole rows.  HBM-bound: 2 rows read, 2 written per
//     kept position and kv-head.  It brings their weights, too.  8192 positions of
//     each of 16 contexts, 8 kv-heads of 128, bf16: 234 us, 4.6 TB/s (a copy of
//     2 GiB 4.9).  In 4-bit pages 115 us (2.5 TB/s): rows of 64 bytes leave half of the
//     lanes without a piece, and scales move a byte at a time.
#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kSelBins = 2048, kSelCopies = 4;     // counters of a bin, side by side
constexpr int kSelHeld = 640;                      // keys that a wave keeps in LDS (two workgroups fit a CU)

// Unsigned keys in the order of the weights, between 0, for places past the
// end, and kForced: -0 is 0, and a NaN, of either sign, comes after +infinity.
constexpr unsigned kForced = 0xffffffffu;
__device__ __forceinline__ unsigned order_key(float w) {
  const unsigned u = __builtin_bit_cast(unsigned, w + 0.0f);
  const unsigned key = u ^ ((unsigned)((int)u >> 31) | 0x80000000u);   // negative ones inverted, the others above them
  return w != w ? kForced - 1 : key;
}

// BY: weights of a lane that are taken at a time.  2 for short sequences, whose
// waves would pass over 8 where they have one (1000 positions: 8.1 us, with 8
// 10.3; 16 contexts of 8192..65536 positions, 8 kv-heads: 53.7 and 39.7).
template <int BY>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ u32x4 hist[kSelBins];                 // a lane in four counts in each component
  __shared__ unsigned pick[2];                     // bin, count above it
  __shared__ unsigned totals[2][kSelWaves];
  __shared__ unsigned held[kSelWaves][kSelHeld];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % a.num_kv_heads, i = blockIdx.x / a.num_kv_heads;
  const EvictDesc sd = a.seq[i];
  const int L = sd.length, n = sd.keep;
  const int64_t row = (int64_t)sd.seq * a.num_kv_heads + g;
  const float* w = a.weights + row * a.stride;
  int32_t* out = a.positions + row * a.out_stride;
  float* wout = a.weights_out != nullptr ? a.weights_out + row * a.out_stride : nullptr;   // its first n: by move
  for (int64_t x = n + tid; x < a.out_stride; x += kSelThreads) {
    out[x] = -1;
    if (wout != nullptr) wout[x] = 0.f;
  }
  if (L == n) {                                    // everything stays
    for (int p = tid; p < n; p += kSelThreads) out[p] = p;
    return;
  }

  // ---- this wave's positions from, from + 64, ..: `steps` of one each lane
  const int steps = (L + kSelThreads - 1) / kSelThreads;
  const int from = wave * steps * 64 + lane;
  const int end = min(L, (wave + 1) * steps * 64);
  const int lo = a.sinks, hi = L - a.recent;       // positions that compete
  // f(key, position) of all positions of this wave, 64 at a time, in order (past
  // its end with keys 0).  The weights come from the L2 each time (a read of 65536
  // is 2 us; held in registers they spill); what takes time is the instructions for
  // each, so groups that compete as a whole skip the tests for the rest.
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    float next[BY];                                // the group after, in flight (past the end: the last weight)
    auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < BY; ++j) next[j] = w[min(from + (j0 + j) * 64, L - 1)];
    };
    load(0);
    for (int j0 = 0; j0 < steps; j0 += BY) {
      const int p0 = from + j0 * 64;
      const int g0 = __builtin_amdgcn_readfirstlane(p0 - lane), g1 = g0 + BY * 64;   // of the group
      if (g0 >= end) break;
      float raw[BY];
#pragma unroll
      for (int j = 0; j < BY; ++j) raw[j] = next[j];
      load(j0 + BY);
      if (g0 >= lo && g1 <= hi && g1 <= end) {
#pragma unroll
        for (int j = 0; j < BY; ++j) f(order_key(raw[j]), p0 + j * 64);
      } else {
#pragma unroll
        for (int j = 0; j < BY; ++j) {
          const int p = p0 + j * 64;
          f(p >= end ? 0u : p < lo || p >= hi ? kForced : order_key(raw[j]), p);
        }
      }
    }
  };

  // ---- the n-th largest key: larger ones stay, and the first `even` equal to it.
  // The second pass keeps the keys that agree with the first one's digit (`count`
  // of this wave), and how many are above them (`sure`): what follows needs only
  // those, or, where they do not fit, all of the wave's keys again.
  unsigned edge = 0, even = (unsigned)n, sure = 0, count = 0;
  unsigned* list = held[wave];
  unsigned* mine = reinterpret_cast<unsigned*>(hist) + lane % kSelCopies;
  auto again = [&](auto&& f) __attribute__((always_inline)) {
    if (count > kSelHeld) {
      each([&](unsigned u, int) __attribute__((always_inline)) { f(u); });
    } else {
      for (unsigned x = 0; x < count; x += 64) f(x + lane < count ? list[x + lane] : 0u);
    }
  };
  for (int b = tid; b < kSelBins; b += kSelThreads) hist[b] = (u32x4){0u, 0u, 0u, 0u};
  __syncthreads();
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    if (pass == 0) {
      each([&](unsigned u, int) __attribute__((always_inline)) {
        if (u != 0) atomicAdd(&mine[(u >> 21) * kSelCopies], 1u);
      });
    } else if (pass == 1) {
      const unsigned agreed = edge >> 21;
      each([&](unsigned u, int) __attribute__((always_inline)) {
        sure += __builtin_popcountll(__builtin_amdgcn_ballot_w64((u >> 21) > agreed));
        const bool in = (u >> 21) == agreed;
        const uint64_t all = __builtin_amdgcn_ballot_w64(in);
        if (all == 0) return;
        const unsigned place =
            __builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, count));
        if (in) {
          atomicAdd(&mine[(u >> 10 & (kSelBins - 1)) * kSelCopies], 1u);
          if (place < kSelHeld) list[place] = u;
        }
        count += __builtin_popcountll(all);
      });
    } else {
      again([&](unsigned u) __attribute__((always_inline)) {
        if ((u >> 10) == edge >> 10) atomicAdd(&mine[(u & 1023) * kSelCopies], 1u);
      });
    }
    __syncthreads();
    // counts from the largest bin down; thread t holds bins 2047 - 2t and 2046 - 2t,
    // and clears them for the next pass
    u32x4& h0 = hist[kSelBins - 1 - 2 * tid];
    u32x4& h1 = hist[kSelBins - 2 - 2 * tid];
    const unsigned c0 = h0[0] + h0[1] + h0[2] + h0[3], c1 = h1[0] + h1[1] + h1[2] + h1[3];
    h0 = h1 = (u32x4){0u, 0u, 0u, 0u};
    unsigned upto = c0 + c1;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned below = __shfl_up(upto, d);
      if (lane >= d) upto += below;
    }
    if (lane == 63) totals[0][wave] = upto;
    __syncthreads();
    for (int x = 0; x < wave; ++x) upto += totals[0][x];
    const unsigned before = upto - c0 - c1;
    if (before < even && before + c0 >= even) pick[0] = kSelBins - 1 - 2 * tid, pick[1] = before;
    else if (before + c0 < even && upto >= even) pick[0] = kSelBins - 2 - 2 * tid, pick[1] = before + c0;
    __syncthreads();
    edge |= pick[0] << shift;
    even -= pick[1];
  }

  // ---- the places of what stays: what the waves before this one keep, then ballots
  unsigned s = count > kSelHeld ? 0 : sure, e = 0;
  again([&](unsigned u) __attribute__((always_inline)) {
    s += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u > edge));
    e += __builtin_popcountll(__builtin_amdgcn_ballot_w64(u == edge));
  });
  __syncthreads();                                 // totals are read
  if (lane == 0) totals[0][wave] = s, totals[1][wave] = e;
  __syncthreads();
  s = e = 0;
  for (int x = 0; x < wave; ++x) s += totals[0][x], e += totals[1][x];
  each([&](unsigned u, int p) __attribute__((always_inline)) {
    const uint64_t above = __builtin_amdgcn_ballot_w64(u > edge), equal = __builtin_amdgcn_ballot_w64(u == edge);
    if ((above | equal) == 0) return;
    const unsigned sb = __builtin_amdgcn_mbcnt_hi((unsigned)(above >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)above, s));
    const unsigned eb =
        __builtin_amdgcn_mbcnt_hi((unsigned)(equal >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)equal, e));
    if (u > edge || (u == edge && eb < even)) out[sb + min(eb, even)] = p;
    s += __builtin_popcountll(above), e += __builtin_popcountll(equal);
  });
}

// A page of targets per workgroup and kv-head.  Rows are ROW bytes of 16-byte
// pieces; 4-bit rows are their codes, and their scales go apart.
template <int ROW, int SCALE>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a) {
  constexpr int kPieces = ROW / 16;
  constexpr int64_t kPage = kBlock * (ROW + SCALE);
  const int hkv = a.num_kv_heads;
  const int block = (int)blockIdx.x + a.first_block;
  const int g = block % hkv;
  const int unit = block / hkv;
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const EvictDesc sd = a.seq[si];
  const int page = unit - a.unit_begin[si];
  const int32_t to = a.to_table[(int64_t)sd.seq * a.to_max_blocks + page];
  const int32_t* from = a.positions + ((int64_t)sd.seq * hkv + g) * a.out_stride + page * kBlock;
  const int32_t* bt = a.block_table + (int64_t)sd.seq * a.max_blocks;
  const int rows = min(kBlock, sd.keep - page * kBlock);
  const int64_t dst = ((int64_t)to * hkv + g) * kPage;
  if (a.weights_out != nullptr && threadIdx.x < rows) {
    const int64_t row = (int64_t)sd.seq * hkv + g;
    a.weights_out[row * a.out_stride + page * kBlock + threadIdx.x] = a.weights[row * a.stride + from[threadIdx.x]];
  }
  if (to < 0 || (int64_t)to >= a.num_blocks) return;   // skipped, as an append's
  auto source = [&](int i, int& slot) __attribute__((always_inline)) {
    const int pos = from[i];
    const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
    const uint32_t id = min((uint32_t)bt[pos / kBlock], nb_max);
    slot = pos % kBlock;
    return ((int64_t)id * hkv + g) * kPage;
  };
  for (int x = threadIdx.x; x < rows * kPieces * 2; x += 256) {
    const bool is_v = x >= rows * kPieces;
    const int y = is_v ? x - rows * kPieces : x;
    const int i = y / kPieces, piece = y % kPieces;
    int slot;
    const int64_t src = source(i, slot);
    char* pool = reinterpret_cast<char*>(is_v ? a.v_pool : a.k_pool);
    const u32x4 val = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pool + src + slot * ROW + piece * 16));
    *reinterpret_cast<u32x4*>(pool + dst + i * ROW + piece * 16) = val;
  }
  if constexpr (SCALE > 0) {
    for (int x = threadIdx.x; x < rows * SCALE * 2; x += 256) {
      const bool is_v = x >= rows * SCALE;
      const int y = is_v ? x - rows * SCALE : x;
      const int i = y / SCALE, piece = y % SCALE;
      int slot;
      const int64_t src = source(i, slot);
      char* pool = reinterpret_cast<char*>(is_v ? a.v_pool : a.k_pool);
      pool[dst + kBlock * ROW + i * SCALE + piece] = pool[src + kBlock * ROW + slot * SCALE + piece];
    }
  }
}

}  // namespace

hipError_t launch_evict_select(const EvictArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.nseq * a.num_kv_heads), block(kSelThreads);
  if (a.seq[0].length <= 4 * kSelThreads) hipLaunchKernelGGL((evict_select_kernel<2>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((evict_select_kernel<8>), grid, block, 0, stream, a);   // longest first
  return hipGetLastError();
}

hipError_t launch_evict_move(const EvictArgs& a, int format, int head_dim, int blocks, hipStream_t stream) {
  const dim3 g(blocks), b(256);
  const bool wide = head_dim == 128;
  if (format == 0 && wide) hipLaunchKernelGGL((evict_move_kernel<256, 0>), g, b, 0, stream, a);
  else if (format == 0) hipLaunchKernelGGL((evict_move_kernel<128, 0>), g, b, 0, stream, a);
  else if (format == 1 && wide) hipLaunchKernelGGL((evict_move_kernel<512, 0>), g, b, 0, stream, a);
  else if (format == 1) hipLaunchKernelGGL((evict_move_kernel<256, 0>), g, b, 0, stream, a);
  else if (wide) hipLaunchKernelGGL((evict_move_kernel<64, 4>), g, b, 0, stream, a);
  else hipLaunchKernelGGL((evict_move_kernel<32, 2>), g, b, 0, stream, a);
  return hipGetLastError();
}

}  // namespace kvt
