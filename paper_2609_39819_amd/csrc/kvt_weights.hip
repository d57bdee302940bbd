// Attention weight of every cached position, gfx950.
//
//   w[b][g][j] (+)= sum over the new rows (token i, head h of kv-head g) that
//                   see j of exp(scale <q_i,h, K_j> - lse_i,h)
// with the log-sum-exp that the attention call returned: half of its products,
// K once and no V.  Every weight is summed by one workgroup in a fixed order.
// Scores are fp32 sums of exact products: bf16 and 4-bit keys are bf16
// operands; fp32 ones three bf16 terms, whose products with a query's three
// are the six that reach 2^-24.
//
// Two kernels, by the rows that the largest sequence adds:
//   * step (at most 32 rows, a decoding step): HBM-bound on K.  4 waves stream
//     32-key tiles from HBM into their operands (no LDS), 16 or 32 rows by
//     v_mfma_f32_16x16x32_bf16;
//   * turn: bound by the exponentials (a score costs 16 cycles of a wave's
//     vector unit for 64 of them and 4 of the matrix unit's).  A workgroup holds 64
//     keys (fp32: 32) as operands in every wave's registers, the waves take
//     the row blocks of 32 in turn, their sums meet in LDS at the end.
#include <type_traits>

#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

template <int FORMAT>
constexpr int kKeyTerms = FORMAT == 1 ? 3 : 1;

// s += K Q^T over the terms of both whose product counts
template <int KN, int QN>
__device__ __forceinline__ void products16(f32x4& s, const bf16x8 (&k)[KN], const bf16x8 (&q)[QN]) {
#pragma unroll
  for (int i = 0; i < KN; ++i)
#pragma unroll
    for (int j = 0; j < QN; ++j)
      if (i + j < 3) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i], q[j], s, 0, 0, 0);
}
template <int KN, int QN>
__device__ __forceinline__ void products32(f32x16& s, const bf16x8 (&k)[KN], const bf16x8 (&q)[QN]) {
#pragma unroll
  for (int i = 0; i < KN; ++i)
#pragma unroll
    for (int j = 0; j < QN; ++j)
      if (i + j < 3) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i], q[j], s, 0, 0, 0);
}

// Sums of v[0 .. N) over the N lanes (two N: N = 16 over 32 lanes) that differ
// in the low bits: on return lane l holds the sum of v[index], the bits of
// index being those of l from `top` down.
template <int N>
__device__ __forceinline__ float scatter_sum(float (&v)[N], int lane, int top) {
#pragma unroll
  for (int n = N / 2, d = top; n > 0; n >>= 1, d >>= 1) {
    const bool up = (lane & d) != 0;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float mine = up ? v[i + n] : v[i], other = up ? v[i] : v[i + n];
      v[i] = mine + __shfl_xor(other, d);
    }
  }
  return v[0];
}

// Old weights are those of the reused positions; the new ones have none.
__device__ __forceinline__ void put(float* w, int key, const SeqDesc& sd, float sum) {
  w[key] = key < sd.prefix ? w[key] + sum : sum;
}

template <typename T, int D, int FORMAT, int NB>
__global__ __launch_bounds__(256, 2) void weights_step_kernel(const WeightsArgs a) {
  constexpr bool kCodes = FORMAT == kMx;
  constexpr int QN = kTerms<T>, KN = kKeyTerms<FORMAT>;
  constexpr int KS = D / 32;
  constexpr int kTK = 32;
  constexpr int kPieces = kCodes ? 1 : FORMAT == 0 ? KS : 2 * KS;   // 16-byte loads per page and lane
  constexpr int64_t kPage = kCodes ? mx_page_bytes(D) : (int64_t)kBlock * D * (FORMAT == 0 ? 2 : 4);
  constexpr int DEPTH = FORMAT == 1 ? 1 : 2;     // tiles in flight
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, qd = lane >> 4;

  const int hkv = a.num_kv_heads, G = a.group;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const int si = unit / a.nsplit, split = unit - si * a.nsplit;
  const SeqDesc sd = a.seq[si];
  const int P = sd.prefix, L = P + sd.suffix, rows = sd.suffix * G;
  const int nblk = (L + kBlock - 1) / kBlock, ntk = (L + kTK - 1) / kTK;
  const int per_split = (ntk + a.nsplit - 1) / a.nsplit;
  const int j0 = split * per_split, j1 = min(ntk, j0 + per_split);
  const int nt = j1 - j0 > wave ? (j1 - j0 - wave + 3) / 4 : 0;

  // ---- this lane's query rows; rows past the last see nothing
  bf16x8 qreg[NB][KS][QN];
  float lse2[NB];
  int lim[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int r = min(b * 16 + l16, rows - 1), t = r / G;
    const int64_t row = (int64_t)(sd.row_off + t) * a.num_q_heads + g * G + (r - t * G);
    const T* qp = reinterpret_cast<const T*>(a.q) + row * D;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) load_terms(qp + (kCodes ? qd * (D / 4) + kk * 8 : kk * 32 + qd * 8), qreg[b][kk]);
    lse2[b] = a.lse[row] * kLog2e;
    lim[b] = b * 16 + l16 < rows ? P + t : -1;
  }
  float* w = a.weights + ((int64_t)sd.seq * hkv + g) * a.stride;
  const char* kpool = reinterpret_cast<const char*>(a.k_pool);
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
  auto page_ids = [&](int j, uint32_t (&ids)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = __builtin_amdgcn_readfirstlane(min(j * 2 + p, nblk - 1));
      const uint32_t raw = (uint32_t)bt[page];
      ids[p] = __builtin_amdgcn_readfirstlane(raw > nb_max ? nb_max : raw);
    }
  };
  struct Stage {
    u32x4 k[2][kPieces];
    unsigned char scale[2];
  };
  auto load_tile = [&](int j, const uint32_t (&ids)[2], Stage& st) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = min(j * 2 + p, nblk - 1);
      const int slot = min(l16, L - 1 - page * kBlock);
      const char* at = kpool + ((int64_t)ids[p] * hkv + g) * kPage;
      if constexpr (kCodes) {
        const char* code = at + slot * (D / 2) + qd * (D / 8);
        if constexpr (KS == 4) {
          st.k[p][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(code));
        } else {
          const u32x2 c2 = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(code));
          st.k[p][0] = (u32x4){c2[0], c2[1], 0u, 0u};
        }
        st.scale[p] = (unsigned char)at[mx_code_bytes(D) + slot * (D / 32) + (D == 128 ? qd : qd >> 1)];
      } else {
        constexpr int PER = FORMAT == 0 ? 1 : 2, ES = FORMAT == 0 ? 2 : 4;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
#pragma unroll
          for (int x = 0; x < PER; ++x)
            st.k[p][kk * PER + x] = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4*>(at + (slot * D + kk * 32 + qd * 8) * ES + 16 * x));
      }
    }
  };
  const float c = a.scale_log2;
  auto tile = [&](Stage& st, int kb, auto&& next) __attribute__((always_inline)) {
    f32x4 s[NB][2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b][p] = (f32x4){0.f, 0.f, 0.f, 0.f};
      const float scale = kCodes ? mx_scale(st.scale[p]) : 0.f;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        bf16x8 kf[KN];
        if constexpr (kCodes) kf[0] = mx_values(st.k[p][0][kk], scale);
        else if constexpr (FORMAT == 0) kf[0] = __builtin_bit_cast(bf16x8, st.k[p][kk]);
        else split3(__builtin_bit_cast(f32x4, st.k[p][2 * kk]), __builtin_bit_cast(f32x4, st.k[p][2 * kk + 1]), kf);
#pragma unroll
        for (int b = 0; b < NB; ++b) products16(s[b][p], kf, qreg[b][kk]);
      }
    }
    next();
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = kb + 16 * (e >> 2) + 4 * qd + (e & 3);
      sum[e] = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e >> 2][e & 3], c, -lse2[b]));
        sum[e] += key > lim[b] ? 0.f : p;
      }
    }
    float total = scatter_sum(sum, lane, 8);     // of element (l16 >> 1), half of it
    total += __shfl_xor(total, 1);
    const int e = l16 >> 1, key = kb + 16 * (e >> 2) + 4 * qd + (e & 3);
    if ((lane & 1) == 0 && key < L) put(w, key, sd, total);
  };

  auto jt = [&](int i) { return j0 + wave + 4 * i; };
  Stage st[DEPTH];
  uint32_t ids[2];
  if (nt > 0) {
    page_ids(jt(0), ids);
#pragma unroll
    for (int x = 0; x < DEPTH; ++x) {
      if (x < nt) load_tile(jt(x), ids, st[x]);
      page_ids(jt(x + 1), ids);
    }
  }
  for (int i = 0; i < nt; i += DEPTH)
#pragma unroll
    for (int x = 0; x < DEPTH; ++x)
      if (i + x < nt)
        tile(st[x], jt(i + x) * kTK, [&]() __attribute__((always_inline)) {
          if (i + x + DEPTH < nt) {
            load_tile(jt(i + x + DEPTH), ids, st[x]);
            page_ids(jt(i + x + DEPTH + 1), ids);
          }
        });
}

template <int FORMAT>
constexpr int kTurnBlocks = FORMAT == 1 ? 1 : 2;   // 32-key blocks of a workgroup

template <typename T, int D, int FORMAT>
__global__ __launch_bounds__(512) void weights_turn_kernel(const WeightsArgs a) {
  constexpr bool kCodes = FORMAT == kMx;
  constexpr int QN = kTerms<T>, KN = kKeyTerms<FORMAT>;
  constexpr int KSTEPS = D / 16;
  constexpr int KB = kTurnBlocks<FORMAT>, KEYS = KB * 32;
  constexpr int64_t kPage = kCodes ? mx_page_bytes(D) : (int64_t)kBlock * D * (FORMAT == 0 ? 2 : 4);
  constexpr int QP = (int)sizeof(T) / 2;         // 16-byte pieces of 8 query columns
  __shared__ float red[8][KEYS];
  const int tid = threadIdx.x;
  const int waves = blockDim.x / 64;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, l32 = lane & 31;

  const int hkv = a.num_kv_heads, G = a.group;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const SeqDesc sd = a.seq[si];
  const int P = sd.prefix, L = P + sd.suffix, rows = sd.suffix * G;
  const int kb = (unit - a.unit_begin[si]) * KEYS;
  const int nblk = (L + kBlock - 1) / kBlock;
  // row blocks that see one of the keys
  const int blocks = (rows + 31) / 32;
  const int first = kb > P ? (int)((int64_t)(kb - P) * G / 32) : 0;

  float acc[KB][16];
#pragma unroll
  for (int x = 0; x < KB; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[x][e] = 0.f;

  if (first + wave < blocks) {
    // ---- the keys, as operands
    const char* kpool = reinterpret_cast<const char*>(a.k_pool);
    const int32_t* bt = a.block_table + (int64_t)sd.seq * a.max_blocks;
    const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
    bf16x8 kf[KB][KSTEPS][KN];
#pragma unroll
    for (int x = 0; x < KB; ++x) {
      const int pos = min(kb + x * 32 + l32, L - 1);
      const uint32_t id = min((uint32_t)bt[min(pos / kBlock, nblk - 1)], nb_max);
      const int slot = pos % kBlock;
      const char* at = kpool + ((int64_t)id * hkv + g) * kPage;
      if constexpr (kCodes) {
#pragma unroll
        for (int y = 0; y < D / 64; ++y) {       // 32 columns: four words under one scale
          const u32x4 c4 = *reinterpret_cast<const u32x4*>(at + slot * (D / 2) + hh * (D / 4) + y * 16);
          const float scale = mx_scale((unsigned char)at[mx_code_bytes(D) + slot * (D / 32) + hh * (D / 64) + y]);
#pragma unroll
          for (int i = 0; i < 4; ++i) kf[x][y * 4 + i][0] = mx_values(c4[i], scale);
        }
      } else {
        typedef typename std::conditional<FORMAT == 0, __bf16, float>::type K;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk)
          load_terms(reinterpret_cast<const K*>(at) + slot * D + kk * 16 + hh * 8, kf[x][kk]);
      }
    }
    // ---- row blocks of 32, the next one's queries in flight
    struct Rows {
      u32x4 q[KSTEPS][QP];
      float lse;
      int lim;
    };
    auto load_rows = [&](int rb, Rows& o) __attribute__((always_inline)) {
      const int r = min(rb * 32 + l32, rows - 1), t = r / G;
      const int64_t row = (int64_t)(sd.row_off + t) * a.num_q_heads + g * G + (r - t * G);
      const char* qp = reinterpret_cast<const char*>(reinterpret_cast<const T*>(a.q) + row * D);
#pragma unroll
      for (int kk = 0; kk < KSTEPS; ++kk)
#pragma unroll
        for (int x = 0; x < QP; ++x)
          o.q[kk][x] = *reinterpret_cast<const u32x4*>(
              qp + (kCodes ? hh * (D / 2) + kk * 8 : kk * 16 + hh * 8) * (int)sizeof(T) + 16 * x);
      o.lse = a.lse[row];
      o.lim = rb * 32 + l32 < rows ? P + t : -1;   // rows past the last see nothing
    };
    const float c = a.scale_log2;
    Rows cur;
    load_rows(first + wave, cur);
    for (int rb = first + wave; rb < blocks; rb += waves) {
      f32x16 s[KB];
#pragma unroll
      for (int x = 0; x < KB; ++x) s[x] = (f32x16){};
#pragma unroll
      for (int kk = 0; kk < KSTEPS; ++kk) {
        bf16x8 qf[QN];
        if constexpr (QN == 1) qf[0] = __builtin_bit_cast(bf16x8, cur.q[kk][0]);
        else split3(__builtin_bit_cast(f32x4, cur.q[kk][0]), __builtin_bit_cast(f32x4, cur.q[kk][QP - 1]), qf);
#pragma unroll
        for (int x = 0; x < KB; ++x) products32(s[x], kf[x][kk], qf);
      }
      const float lse2 = cur.lse * kLog2e;
      const int lim = cur.lim;
      if (rb + waves < blocks) load_rows(rb + waves, cur);
      // the block's first row sees the fewest keys; the last block may end early
      const bool whole = P + rb * 32 / G >= kb + KEYS - 1 && rb * 32 + 32 <= rows;
      if (whole) {
#pragma unroll
        for (int x = 0; x < KB; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[x][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], c, -lse2));
      } else {
        const int thr = lim - kb - 4 * hh;       // keys past lim: offset > thr
#pragma unroll
        for (int x = 0; x < KB; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], c, -lse2));
            acc[x][e] += x * 32 + 8 * (e >> 2) + (e & 3) > thr ? 0.f : p;
          }
      }
    }
  }
  // ---- sums over the rows: the lanes of a half, then the waves in order
#pragma unroll
  for (int x = 0; x < KB; ++x) {
    float sum = scatter_sum(acc[x], lane, 16);   // of element l32 >> 1, half of it
    sum += __shfl_xor(sum, 1);
    const int e = l32 >> 1;
    if ((lane & 1) == 0) red[wave][x * 32 + 8 * (e >> 2) + 4 * hh + (e & 3)] = sum;
  }
  __syncthreads();
  for (int k = tid; k < KEYS; k += blockDim.x) {
    if (kb + k >= L) break;
    float sum = 0.f;
    for (int x = 0; x < waves; ++x) sum += red[x][k];
    put(a.weights + ((int64_t)sd.seq * hkv + g) * a.stride, kb + k, sd, sum);
  }
}

template <typename T, int D, int FORMAT>
void launch_step_as(const WeightsArgs& a, int grid, hipStream_t stream) {
  int rows = 0;
  for (int i = 0; i < a.nseq; ++i) rows = a.seq[i].suffix * a.group > rows ? a.seq[i].suffix * a.group : rows;
  if (rows <= 16) hipLaunchKernelGGL((weights_step_kernel<T, D, FORMAT, 1>), dim3(grid), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((weights_step_kernel<T, D, FORMAT, 2>), dim3(grid), dim3(256), 0, stream, a);
}
template <typename T, int D, int FORMAT>
void launch_turn_as(const WeightsArgs& a, int waves, int grid, hipStream_t stream) {
  hipLaunchKernelGGL((weights_turn_kernel<T, D, FORMAT>), dim3(grid), dim3(64 * waves), 0, stream, a);
}

}  // namespace

int weights_keys_per_unit(int format) { return 32 * (format == 1 ? kTurnBlocks<1> : kTurnBlocks<0>); }

hipError_t launch_weights_step(const WeightsArgs& a, int format, int dtype, int head_dim, int grid, hipStream_t stream) {
  const bool wide = head_dim == 128;
  if (format == 0) wide ? launch_step_as<__bf16, 128, 0>(a, grid, stream) : launch_step_as<__bf16, 64, 0>(a, grid, stream);
  else if (format == 1) wide ? launch_step_as<float, 128, 1>(a, grid, stream) : launch_step_as<float, 64, 1>(a, grid, stream);
  else if (dtype == 0) wide ? launch_step_as<__bf16, 128, kMx>(a, grid, stream) : launch_step_as<__bf16, 64, kMx>(a, grid, stream);
  else wide ? launch_step_as<float, 128, kMx>(a, grid, stream) : launch_step_as<float, 64, kMx>(a, grid, stream);
  return hipGetLastError();
}

hipError_t launch_weights_turn(const WeightsArgs& a, int format, int dtype, int head_dim, int waves, int grid,
                               hipStream_t stream) {
  const bool wide = head_dim == 128;
  if (format == 0) wide ? launch_turn_as<__bf16, 128, 0>(a, waves, grid, stream) : launch_turn_as<__bf16, 64, 0>(a, waves, grid, stream);
  else if (format == 1) wide ? launch_turn_as<float, 128, 1>(a, waves, grid, stream) : launch_turn_as<float, 64, 1>(a, waves, grid, stream);
  else if (dtype == 0) wide ? launch_turn_as<__bf16, 128, kMx>(a, waves, grid, stream) : launch_turn_as<__bf16, 64, kMx>(a, waves, grid, stream);
  else wide ? launch_turn_as<float, 128, kMx>(a, waves, grid, stream) : launch_turn_as<float, 64, kMx>(a, waves, grid, stream);
  return hipGetLastError();
}

}  // namespace kvt
