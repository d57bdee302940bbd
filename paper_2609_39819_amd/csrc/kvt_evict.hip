// Eviction by accumulated weight, gfx950.
//
// Per sequence and kv-head, of L positions n = min(L, keep) stay: the first
// `sinks`, the last `recent`, and of those between them the heaviest, of equal
// ones the lowest positions.  Two launches:
//   * select: one workgroup per (sequence, kv-head).  The k-th largest weight is
//     found as a 32-bit key, 8 bits at a time from the top: a histogram of the
//     keys that agree so far (integer counts in LDS, so their order does not
//     matter), then the bin that holds the k-th.  Then the positions are taken in
//     order: a scan counts those that stay, and gives each its place.
//   * move: the kept rows into the other pages, 16 bytes a lane in the order of
//     the targets; reads are whole rows.  HBM-bound: 2 rows read, 2 written per
//     kept position and kv-head.
#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kPer = 4;                            // neighbouring positions of one thread

// Unsigned keys in the order of the weights; -0 is 0, and a NaN, of either sign,
// comes after +infinity.
__device__ __forceinline__ unsigned order_key(float w) {
  const unsigned u = __builtin_bit_cast(unsigned, w + 0.0f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ unsigned hist[kSelWaves][256];        // one per wave: fewer lanes on one counter
  __shared__ unsigned pick[2];                     // bin, counts above it
  __shared__ unsigned totals[2][kSelWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x % a.num_kv_heads, i = blockIdx.x / a.num_kv_heads;
  const EvictDesc sd = a.seq[i];
  const int L = sd.length, n = sd.keep;
  const int64_t row = (int64_t)sd.seq * a.num_kv_heads + g;
  const float* w = a.weights + row * a.stride;
  int32_t* out = a.positions + row * a.out_stride;
  float* wout = a.weights_out != nullptr ? a.weights_out + row * a.out_stride : nullptr;
  const int lo = L > n ? a.sinks : L, hi = L > n ? L - a.recent : L;   // positions that compete

  // ---- the border: keys above `edge` stay, and the first `even` equal to it
  unsigned edge = 0, even = 0;
  int k = n - (L - (hi - lo));                     // how many of them stay
  if (L > n && k > 0) {
    unsigned want = (unsigned)k;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int b = tid; b < kSelWaves * 256; b += kSelThreads) (&hist[0][0])[b] = 0;
      __syncthreads();
      for (int p = lo + tid; p < hi; p += kSelThreads) {
        const unsigned u = order_key(w[p]);
        if (shift == 24 || (u >> (shift + 8)) == (edge >> (shift + 8))) atomicAdd(&hist[wave][(u >> shift) & 255], 1u);
      }
      __syncthreads();
      // counts from the largest bin down; thread t holds bin 255 - t
      unsigned count = 0;
      if (tid < 256) {
#pragma unroll
        for (int x = 0; x < kSelWaves; ++x) count += hist[x][255 - tid];
      }
      unsigned upto = count;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned below = __shfl_up(upto, d);
        if (lane >= d) upto += below;
      }
      if (tid < 256 && lane == 63) totals[0][wave] = upto;
      __syncthreads();
      if (tid < 256) {
        for (int x = 0; x < wave; ++x) upto += totals[0][x];
        if (upto >= want && upto - count < want) pick[0] = 255 - tid, pick[1] = upto - count;
      }
      __syncthreads();
      edge |= pick[0] << shift;
      want -= pick[1];
    }
    even = want;
  }

  // ---- the positions in order.  A thread's count packs what stays for certain
  // and what equals the edge; the latter stay while they are among the first.
  unsigned sure_before = 0, equal_before = 0;      // of the tiles before
  for (int p0 = 0; p0 < L; p0 += kSelThreads * kPer) {
    unsigned sure = 0, equal = 0, mask_sure = 0, mask_equal = 0;
    float val[kPer];
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      const int p = p0 + tid * kPer + x;
      if (p >= L) break;
      val[x] = w[p];
      const unsigned u = order_key(val[x]);
      if (p < lo || p >= hi || (k > 0 && u > edge)) ++sure, mask_sure |= 1u << x;
      else if (k > 0 && u == edge) ++equal, mask_equal |= 1u << x;
    }
    unsigned s = sure, e = equal;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned ps = __shfl_up(s, d), pe = __shfl_up(e, d);
      if (lane >= d) s += ps, e += pe;
    }
    if (lane == 63) totals[0][wave] = s, totals[1][wave] = e;
    __syncthreads();
    unsigned all_s = 0, all_e = 0;
#pragma unroll
    for (int x = 0; x < kSelWaves; ++x) {
      const unsigned ts = totals[0][x], te = totals[1][x];
      if (x < wave) s += ts, e += te;
      all_s += ts, all_e += te;
    }
    __syncthreads();
    s += sure_before - sure, e += equal_before - equal;   // before this thread's first position
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
      const bool is_sure = mask_sure >> x & 1, is_equal = mask_equal >> x & 1;
      if (is_sure || (is_equal && e < even)) {
        const int64_t at = (int64_t)s + min(e, even);
        out[at] = p0 + tid * kPer + x;
        if (wout != nullptr) wout[at] = val[x];
      }
      s += is_sure, e += is_equal;
    }
    sure_before += all_s, equal_before += all_e;
  }
  for (int64_t x = n + tid; x < a.out_stride; x += kSelThreads) {
    out[x] = -1;
    if (wout != nullptr) wout[x] = 0.f;
  }
}

// A page of targets per workgroup and kv-head.  Rows are ROW bytes of 16-byte
// pieces; 4-bit rows are their codes, and their scales go apart.
template <int ROW, int SCALE>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a) {
  constexpr int kPieces = ROW / 16;
  constexpr int64_t kPage = kBlock * (ROW + SCALE);
  const int hkv = a.num_kv_heads;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const EvictDesc sd = a.seq[si];
  const int page = unit - a.unit_begin[si];
  const int32_t to = a.to_table[(int64_t)sd.seq * a.to_max_blocks + page];
  if (to < 0 || (int64_t)to >= a.num_blocks) return;   // skipped, as an append's
  const int32_t* from = a.positions + ((int64_t)sd.seq * hkv + g) * a.out_stride + page * kBlock;
  const int32_t* bt = a.block_table + (int64_t)sd.seq * a.max_blocks;
  const int rows = min(kBlock, sd.keep - page * kBlock);
  const int64_t dst = ((int64_t)to * hkv + g) * kPage;
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
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)a.nseq * a.num_kv_heads), dim3(kSelThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_evict_move(const EvictArgs& a, int format, int head_dim, int grid, hipStream_t stream) {
  const dim3 g(grid), b(256);
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
