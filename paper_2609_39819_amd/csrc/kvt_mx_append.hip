// Rows of new tokens into 4-bit pages, and their values back.
//
// A row's D columns are held in groups of 32: one byte s for the power of two
// 2^e, e = s - 127, and a 4-bit code (e2m1: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and
// their negatives) for every x / 2^e, rounded to nearest with ties to the even
// code.  e is the least with max |x| <= 7 * 2^e: values up to 7 round to 6, off
// by no more than the largest step's half, so a larger e would only coarsen
// the grid.  e is held in -125 .. 96: every value is a normal bf16 number, and
// a sum of 2^20 of them with weights up to 2^8 stays in fp32's range.
//
// Both kernels are HBM-bound scatters: a lane takes 8 columns of K and of V (a
// group is four lanes, whose maximum meets through cross-lane moves), so a
// row's 16 lanes (D = 128) read 256 contiguous bytes and write 64.  14336 tokens
// of 8 kv-heads of 128, bf16, 74 MB: written in 18.5 us (4.0 TB/s), read back in
// 13.5 (5.5; a copy of 2 GiB reaches 4.9).  With a workgroup's lanes along the heads
// of two tokens instead, the lines of a page's scales went to several XCDs: 19.8
// and 16.1 us, 35 MB read for 16.  256 single tokens: 3.5 us each, a launch.
#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

// Index of the launch-local sequence that owns packed row r.  As many rows as
// sequences: one each, no search.
__device__ __forceinline__ int owner(const MxRowsArgs& a, int32_t row) {
  if (a.rows == a.nseq) return row - a.row_begin;
  int lo = 0, hi = a.nseq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seq[mid].row_off <= row) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One lane's piece: token row, kv-head and first column of 8, and its page.  A
// workgroup takes consecutive rows of one kv-head, 16 (D = 128) or 32, so that a
// page's lines, its scales' above all, are used at once.
struct Piece {
  int32_t row, g, c, slot;
  int64_t page;   // -1: an id outside the pool
};
template <int D>
constexpr int kRows = 256 / (D / 8);
template <int D>
__device__ __forceinline__ bool piece_of(const MxRowsArgs& a, int32_t unit, Piece& p) {
  const int32_t r = unit / a.num_kv_heads * kRows<D> + (int32_t)threadIdx.x / (D / 8);
  if (r >= a.rows) return false;   // a row's lanes are in or out together
  p.row = a.row_begin + r;
  p.g = unit % a.num_kv_heads;
  p.c = threadIdx.x % (D / 8);
  const SeqDesc sd = a.seq[owner(a, p.row)];
  const int32_t pos = sd.prefix + (p.row - sd.row_off);
  const int32_t id = a.block_table[(int64_t)sd.seq * a.max_blocks + pos / kBlock];
  p.page = id < 0 || (int64_t)id >= a.num_blocks ? -1 : id;
  p.slot = pos % kBlock;
  return true;
}

template <int D>
__host__ __device__ int64_t units_of(const MxRowsArgs& a) {
  return (int64_t)((a.rows + kRows<D> - 1) / kRows<D>) * a.num_kv_heads;
}
constexpr int64_t kMostBlocks = 1 << 20;

struct Eight {
  float x[8];
};
__device__ __forceinline__ Eight load_eight(const __bf16* p) {
  const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    e.x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    e.x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
  return e;
}
__device__ __forceinline__ Eight load_eight(const float* p) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
  return Eight{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}

// Scale byte of a group of 32 (four lanes), and this lane's 8 codes; `bad` if
// one of this lane's values is no number.  The largest magnitude is compared
// by its bits: 7 * 2^e has the fraction 0x600000 under the exponent e + 2.
__device__ __forceinline__ unsigned quantise(const Eight& e, unsigned& scale, bool& bad) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(unsigned, e.x[i]) & 0x7fffffffu);
  bad = top >= 0x7f800000u;
  top = max(top, (unsigned)__shfl_xor((int)top, 1));
  top = max(top, (unsigned)__shfl_xor((int)top, 2));
  const int byte = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  scale = (unsigned)min(max(byte, 127 - 125), 127 + 96);
  const float s = mx_scale(scale);
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[0], e.x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[2], e.x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[4], e.x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e.x[6], e.x[7], s, 3);
  return w;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void mx_append_kernel(const MxRowsArgs a) {
  constexpr int kLanes = D / 8;
  constexpr int64_t kPage = mx_page_bytes(D);
  for (int64_t unit = blockIdx.x; unit < units_of<D>(a); unit += gridDim.x) {
    Piece p;
    if (!piece_of<D>(a, (int32_t)unit, p)) continue;
    const int64_t col = (int64_t)p.g * D + p.c * 8;
    const Eight k = load_eight(reinterpret_cast<const T*>(a.k) + p.row * a.k_stride + col);
    const Eight v = load_eight(reinterpret_cast<const T*>(a.v) + p.row * a.v_stride + col);
    unsigned ks, vs;
    bool kbad, vbad;
    const unsigned kw = quantise(k, ks, kbad), vw = quantise(v, vs, vbad);
    // one such value in K or V marks the token for this kv-head
    const uint64_t bad = __builtin_amdgcn_ballot_w64(kbad || vbad);
    const uint64_t mine = ((1ull << kLanes) - 1) << (threadIdx.x & 63 & ~(kLanes - 1));
    if (bad & mine) ks = vs = kMxNan;
    if (p.page < 0) continue;
    const int64_t at = (p.page * a.num_kv_heads + p.g) * kPage;
    char* kp = reinterpret_cast<char*>(a.k_pool) + at;
    char* vp = reinterpret_cast<char*>(a.v_pool) + at;
    const int code = p.slot * (D / 2) + p.c * 4;
    *reinterpret_cast<unsigned*>(kp + code) = kw;
    *reinterpret_cast<unsigned*>(vp + code) = vw;
    if (p.c % 4 == 0) {
      const int scale = mx_code_bytes(D) + p.slot * (D / 32) + p.c / 4;
      kp[scale] = (char)ks;
      vp[scale] = (char)vs;
    }
  }
}

__device__ __forceinline__ void store_eight(__bf16* p, bf16x8 x) {
  *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, x);
}
__device__ __forceinline__ void store_eight(float* p, bf16x8 x) {
  const u32x4 w = __builtin_bit_cast(u32x4, x);
  u32x4 lo, hi;
  lo[0] = w[0] << 16, lo[1] = w[0] & 0xffff0000u, lo[2] = w[1] << 16, lo[3] = w[1] & 0xffff0000u;
  hi[0] = w[2] << 16, hi[1] = w[2] & 0xffff0000u, hi[2] = w[3] << 16, hi[3] = w[3] & 0xffff0000u;
  *reinterpret_cast<u32x4*>(p) = lo;
  *reinterpret_cast<u32x4*>(p + 4) = hi;
}

// A block id outside the pool reads the last page (the values are then
// unspecified).
template <typename T, int D>
__global__ __launch_bounds__(256) void mx_read_kernel(const MxRowsArgs a) {
  constexpr int64_t kPage = mx_page_bytes(D);
  for (int64_t unit = blockIdx.x; unit < units_of<D>(a); unit += gridDim.x) {
    Piece p;
    if (!piece_of<D>(a, (int32_t)unit, p)) continue;
    const int64_t page = p.page < 0 ? a.num_blocks - 1 : p.page;
    const int64_t at = (page * a.num_kv_heads + p.g) * kPage;
    const char* kp = reinterpret_cast<const char*>(a.k_pool) + at;
    const char* vp = reinterpret_cast<const char*>(a.v_pool) + at;
    const int code = p.slot * (D / 2) + p.c * 4, scale = mx_code_bytes(D) + p.slot * (D / 32) + p.c / 4;
    const unsigned kw = *reinterpret_cast<const unsigned*>(kp + code), vw = *reinterpret_cast<const unsigned*>(vp + code);
    const float ks = mx_scale((unsigned char)kp[scale]), vs = mx_scale((unsigned char)vp[scale]);
    const int64_t col = (int64_t)p.g * D + p.c * 8;
    store_eight(reinterpret_cast<T*>(a.k) + p.row * a.k_stride + col, mx_values(kw, ks));
    store_eight(reinterpret_cast<T*>(a.v) + p.row * a.v_stride + col, mx_values(vw, vs));
  }
}

unsigned blocks_for(const MxRowsArgs& a, int head_dim) {
  const int64_t units = head_dim == 128 ? units_of<128>(a) : units_of<64>(a);
  return (unsigned)(units > kMostBlocks ? kMostBlocks : units);   // grid-stride beyond
}

}  // namespace

hipError_t launch_mx_append(const MxRowsArgs& a, int dtype, int head_dim, hipStream_t stream) {
  const dim3 grid(blocks_for(a, head_dim)), block(256);
  if (dtype == 0 && head_dim == 128) hipLaunchKernelGGL((mx_append_kernel<__bf16, 128>), grid, block, 0, stream, a);
  else if (dtype == 0 && head_dim == 64) hipLaunchKernelGGL((mx_append_kernel<__bf16, 64>), grid, block, 0, stream, a);
  else if (dtype == 1 && head_dim == 128) hipLaunchKernelGGL((mx_append_kernel<float, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((mx_append_kernel<float, 64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_mx_read(const MxRowsArgs& a, int dtype, int head_dim, hipStream_t stream) {
  const dim3 grid(blocks_for(a, head_dim)), block(256);
  if (dtype == 0 && head_dim == 128) hipLaunchKernelGGL((mx_read_kernel<__bf16, 128>), grid, block, 0, stream, a);
  else if (dtype == 0 && head_dim == 64) hipLaunchKernelGGL((mx_read_kernel<__bf16, 64>), grid, block, 0, stream, a);
  else if (dtype == 1 && head_dim == 128) hipLaunchKernelGGL((mx_read_kernel<float, 128>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((mx_read_kernel<float, 64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace kvt
