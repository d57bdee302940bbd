// Rotary positions, by themselves and on the way into the cache pages.
//
// Column pairs (a, b) of a query or key row turn by an angle that grows with
// the row's position: with theta = position * inv_freq,
//   a' = a cos(theta) - b sin(theta),   b' = b cos(theta) + a sin(theta).
// The pairs are columns (j, j + R/2) of each rotated run of R columns, or the
// neighbours (2j, 2j + 1); each frequency reads the position of its own axis
// (time, height, width of an image patch); columns past R and V rows are
// copied bit for bit.
//
// Angles.  theta is needed modulo one turn, and far positions make it large:
// 131071 * 1 rad in fp32 is off by up to 2^-8 rad.  The host turns each
// frequency into turns per position in fp64, the kernel multiplies by the
// position and takes off the whole turns in fp64 (three roundings of 2^-53 of the
// turns: under 2^-23 turns at one radian per position and the largest position
// there is); only the rest becomes fp32 (2^-26 turns), and its sine and cosine are
// those of sincospif.  The rotation is fp32, rounded once to the storage type.
//
// One launch moves q, K and V of a token.  The lanes of a token form its sines and
// cosines between them, share them through LDS, keep those of their own columns in
// registers and take two rows each, all in flight at once: a workgroup reads and
// writes whole tokens, about 24 KB of consecutive bytes each way.  (Eight heads of
// four tokens at a time, four rows in flight per lane: 14336 tokens behind a fused
// projection, 96/8 heads, 162.5 us, 139.4 so; 24576 tokens of 24 heads 55.2 and
// 52.9, inputs not in a cache.)  Bound by HBM: 5.9 and 5.7 TB/s in these two, a plain
// copy of as many bytes 5.4; by the launch for a decoding step.
#include <algorithm>

#include "kvt_device.h"
#include "kvt_rotary.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kThreads = 512;
constexpr int kAhead = 2;   // heads per lane whose loads are in flight together

// Eight consecutive elements of a row, as stored.
template <typename T>
struct Piece {
  u32x4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const T* p) {
  Piece<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i)
    r.w[i] = reinterpret_cast<const u32x4*>(p)[i];
  return r;
}
// bf16 pieces go out with the nontemporal policy (24576 tokens of 24 heads of 128:
// 55.7 us without, 52.8 with); an fp32 piece is two stores that share 32 bytes,
// which need the cache to join them (8192 tokens of 32/8 heads of 64: 34.4 and
// 42.4 us).  Loads are ordinary ones (nontemporal 10 % slower).
template <typename T>
__device__ __forceinline__ void store_piece(T* p, const Piece<T>& x) {
  if constexpr (sizeof(T) == 2) {
    __builtin_nontemporal_store(x.w[0], reinterpret_cast<u32x4*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<u32x4*>(p)[i] = x.w[i];
  }
}
__device__ __forceinline__ void widen(const Piece<__bf16>& x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __builtin_bit_cast(float, x.w[0][i] << 16);
    f[2 * i + 1] = __builtin_bit_cast(float, x.w[0][i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const Piece<float>& x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned u = x.w[i / 4][i % 4];
    f[i] = __builtin_bit_cast(float, u);
  }
}
__device__ __forceinline__ void narrow(const float (&f)[8], Piece<__bf16>& x) {
  x.w[0] = round8((f32x4){f[0], f[1], f[2], f[3]}, (f32x4){f[4], f[5], f[6], f[7]});
}
__device__ __forceinline__ void narrow(const float (&f)[8], Piece<float>& x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x.w[i / 4][i % 4] = __builtin_bit_cast(unsigned, f[i]);
}

// A lane's pieces of a row: two runs of eight columns, first and second.  In a
// rotated run of R columns they are R/2 apart, so that eight columns of the one
// are the partners of eight of the other (split pairs) or both hold whole pairs
// (neighbours); either way consecutive lanes read consecutive bytes.
template <typename T, int D, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  constexpr int SLOTS = D / 16;                            // lanes per row
  __shared__ float2 table[kThreads / SLOTS * (D / 2)];     // cosine and sine of (token, frequency)
  const int hl_count = a.head_lanes;                       // a power of two
  const int slot = threadIdx.x % SLOTS;
  const int hl = threadIdx.x / SLOTS & (hl_count - 1);
  const int lanes = SLOTS * hl_count;                      // lanes per token
  const int token = threadIdx.x / lanes;
  const int64_t r = min((int64_t)blockIdx.x * (kThreads / lanes) + token, a.rows - 1);   // launch-local row
  const bool live = (int64_t)blockIdx.x * (kThreads / lanes) + token < a.rows;
  const int64_t row = a.row_begin + r;                     // packed row of the call
  const int hq = a.num_q_heads, hkv = a.num_kv_heads;
  const int jobs = hq + 2 * hkv;                           // q rows, K rows, V rows of one token

  // ---- where the token's K/V go, and its position
  int64_t page_row = -1;    // row of (page, head 0, slot) in the pools, -1: nowhere
  int32_t logical = 0;
  if (hkv > 0) {
    int lo = 0, hi = a.nseq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.seq[mid].row_off <= row) lo = mid;
      else hi = mid - 1;
    }
    const SeqDesc sd = a.seq[lo];
    logical = sd.prefix + (int32_t)(row - sd.row_off);
    const int32_t bid = a.block_table[(int64_t)sd.seq * a.max_blocks + logical / kBlock];
    if (bid >= 0 && (int64_t)bid < a.num_blocks) page_row = (int64_t)bid * hkv * kBlock + logical % kBlock;
  }

  // ---- the token's sines and cosines
  const int width = D / a.parts, rot = a.rot_dim, pairs = rot / 2;
  for (int f = threadIdx.x % lanes; f < pairs; f += lanes) {
    const int32_t pos = a.positions ? a.positions[(int64_t)a.axis[f] * a.total_rows + row] : logical;
    double t = (double)pos * a.turns[f];
    t -= __builtin_rint(t);
    float sn, cs;
    sincospif(2.0f * (float)t, &sn, &cs);
    table[token * pairs + f] = make_float2(cs, sn);
  }
  __syncthreads();
  if (!live) return;

  // ---- the lane's columns of a rotated row, and their sines and cosines
  const int part = slot / (width / 16), u = slot % (width / 16);
  const bool turns = u < rot / 16;
  const int col0 = part * width + (turns ? 8 * u : rot + 8 * (u - rot / 16));
  const int col1 = col0 + (turns ? rot : width - rot) / 2;
  float cs[8], sn[8];
  if (turns) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // split pairs: frequencies 8u .. 8u+7 turn both runs; neighbours: four each
      const int f = PAIRS ? (i < 4 ? 4 * u + i : rot / 4 + 4 * u + i - 4) : 8 * u + i;
      const float2 e = table[token * pairs + f];
      cs[i] = e.x, sn[i] = e.y;
    }
  }

  // ---- the token's rows, kAhead of this lane's at a time
  const T* q = reinterpret_cast<const T*>(a.q) + row * a.q_stride;
  const T* k = reinterpret_cast<const T*>(a.k_new) + row * a.k_stride;
  const T* v = reinterpret_cast<const T*>(a.v_new) + row * a.v_stride;
  T* qo = reinterpret_cast<T*>(a.q_out) + row * a.q_out_stride;
  const int step = hl_count * gridDim.y;
  for (int j0 = hl + hl_count * blockIdx.y; j0 < jobs; j0 += step * kAhead) {
    Piece<T> p0[kAhead], p1[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int j = j0 + i * step;
      if (j >= jobs) break;
      const bool is_v = j >= hq + hkv;
      const T* src = j < hq ? q + (int64_t)j * D : is_v ? v + (int64_t)(j - hq - hkv) * D : k + (int64_t)(j - hq) * D;
      p0[i] = load_piece(src + (is_v ? 8 * slot : col0));
      p1[i] = load_piece(src + (is_v ? 8 * slot + D / 2 : col1));
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int j = j0 + i * step;
      if (j >= jobs) break;
      const bool is_v = j >= hq + hkv;
      if (turns && !is_v) {
        float x[8], y[8];
        widen(p0[i], x);
        widen(p1[i], y);
        if constexpr (PAIRS) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float c0 = cs[e / 2], s0 = sn[e / 2], c1 = cs[4 + e / 2], s1 = sn[4 + e / 2];
            const float x0 = x[e], x1 = x[e + 1], y0 = y[e], y1 = y[e + 1];
            x[e] = x0 * c0 - x1 * s0;
            x[e + 1] = x1 * c0 + x0 * s0;
            y[e] = y0 * c1 - y1 * s1;
            y[e + 1] = y1 * c1 + y0 * s1;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x0 = x[e], y0 = y[e];
            x[e] = x0 * cs[e] - y0 * sn[e];
            y[e] = y0 * cs[e] + x0 * sn[e];
          }
        }
        narrow(x, p0[i]);
        narrow(y, p1[i]);
      }
      T* dst;
      if (j < hq) {
        dst = qo + (int64_t)j * D;
      } else {
        if (page_row < 0) continue;   // an id outside the pool is never dereferenced
        const int64_t at = (page_row + (int64_t)(is_v ? j - hq - hkv : j - hq) * kBlock) * D;
        dst = reinterpret_cast<T*>(is_v ? a.v_pool : a.k_pool) + at;
      }
      store_piece(dst + (is_v ? 8 * slot : col0), p0[i]);
      store_piece(dst + (is_v ? 8 * slot + D / 2 : col1), p1[i]);
    }
  }
}

template <typename T, int D>
void launch_as(RotaryArgs& a, int cus, hipStream_t stream) {
  const int64_t jobs = a.num_q_heads + 2 * (int64_t)a.num_kv_heads;
  a.head_lanes = 1;   // a token's rows in one go, as far as the workgroup's lanes reach
  while (a.head_lanes * kAhead < jobs && a.head_lanes < kThreads / (D / 16)) a.head_lanes *= 2;
  const int64_t tokens = kThreads / (D / 16 * a.head_lanes);
  const int64_t tiles = (a.rows + tokens - 1) / tokens, steps = (jobs + a.head_lanes - 1) / a.head_lanes;
  // few tokens: the heads are spread over workgroups until there are four per CU
  const int64_t gy = std::max<int64_t>(1, std::min<int64_t>({steps, (4 * (int64_t)cus + tiles - 1) / tiles, 65535}));
  const dim3 grid((unsigned)tiles, (unsigned)gy), block(kThreads);
  if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, D, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((rotary_kernel<T, D, false>), grid, block, 0, stream, a);
}

}  // namespace

hipError_t launch_rotary(RotaryArgs& a, int dtype, int head_dim, int cus, hipStream_t stream) {
  if (dtype == 0 && head_dim == 128) launch_as<__bf16, 128>(a, cus, stream);
  else if (dtype == 0 && head_dim == 64) launch_as<__bf16, 64>(a, cus, stream);
  else if (dtype == 1 && head_dim == 128) launch_as<float, 128>(a, cus, stream);
  else launch_as<float, 64>(a, cus, stream);
  return hipGetLastError();
}

}  // namespace kvt
