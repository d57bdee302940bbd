// Extend attention over 4-bit pages, gfx950.
//
// The formula and the decomposition are kvt_extend.hip's: 256 packed query rows
// per workgroup, 8 waves of 32 rows, 64-key tiles in a double-buffered LDS ring,
// S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16, fp32 online
// softmax in log2 units.  What differs:
//   * a tile arrives as 4-bit codes, 16 bytes a lane: waves 0..3 take a page of K
//     each, waves 4..7 a page of V; a lane has 32 columns of one key under one
//     scale (D = 128) and converts them once, for all 256 rows, into bf16 on the
//     way into LDS.  A tile is loaded two steps ahead of its use and converted
//     one step ahead;
//   * the row sums add the fp32 probabilities, so the log-sum-exp keeps fp32's
//     precision;
//   * fp32 queries and probabilities are three bf16 terms each (the 4-bit
//     values are exact in bf16), three products in place of one.
// Positions past the end of the sequence read the last real position; their
// scores are replaced by -inf.  A token that is not a number counts through K,
// whose score is one for the rows that see it; its V is 0 in LDS, so that the
// other rows of the tile do not take it in with a weight of 0.
//
// Bound by the matrix products, with the exponentials and the conversion of the
// probabilities beside them, as over bf16 pages.  32/8 heads of 128, bf16: 2048
// new tokens over 131072, 3.95 ms (1120 TFLOP/s; over bf16 pages 3.90; products 49 %
// of the SIMDs' cycles, vector instructions 46 %); 512 over 8192, 82 us (89), with
// fp32 queries 170; 8 sequences with heads of 64, 32..128 over 1024..16384, 56 us (57;
// 20 % and 38 %): the products of 64 columns take no longer than the exponentials, and
// the rows of a short message do not fill their tile of 256.  fp32 queries over heads
// of 128 spill 27 registers in the main loop.
#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kThreads = kExtWaves * 64;
constexpr int KT = kExtKeysPerTile;   // 64 keys per tile = 4 pages

template <int D>
struct MxHalfTile {
  __bf16 e[KT * D];
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void mx_extend_kernel(const ExtendArgs a) {
  constexpr int NT = kTerms<T>;
  constexpr int KSTEPS = D / 16;
  constexpr int DT = D / 32;
  constexpr int WORDS = D / 32;                  // words of codes per lane and tile
  constexpr int64_t kPage = mx_page_bytes(D);
  constexpr float kRescaleSlack = 8.0f;
  __shared__ __attribute__((aligned(1024))) MxHalfTile<D> slot0[2];   // K, V
  __shared__ __attribute__((aligned(1024))) MxHalfTile<D> slot1[2];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5;
  const int l32 = lane & 31;

  // ---- which (sequence, kv-head, row tile, key split) this workgroup owns;
  // the longest (last) row tile first
  const int hkv = a.num_kv_heads;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const SeqDesc sd = a.seq[si];
  const int local = unit - a.unit_begin[si];
  const int sets = a.nsplit;
  const int G = a.group;
  const int rows_seq = sd.suffix * G;
  const int ntile = (rows_seq + kExtTileRows - 1) / kExtTileRows;
  const int last = a.last[si];
  const bool last_tile = local < last;
  const int nsplit = last_tile ? last : sets;
  const int rest = last_tile ? local : local - last;
  const int rt = last_tile ? ntile - 1 : ntile - 2 - rest / sets;
  const int split = last_tile ? local : rest % sets;
  const int r0 = rt * kExtTileRows;
  const int P = sd.prefix;
  const int L = P + sd.suffix;
  const int nblk = (L + kBlock - 1) / kBlock;
  const int t_last = min(sd.suffix - 1, (r0 + kExtTileRows - 1) / G);
  const int ntiles_kv = (P + t_last + KT) / KT;
  const int per_split = (ntiles_kv + nsplit - 1) / nsplit;
  const int j0 = split * per_split;
  const int j1 = min(ntiles_kv, j0 + per_split);
  const int lim_min = P + r0 / G;                // smallest last-visible key of the row tile

  // ---- this lane's query row
  int r = r0 + wave * 32 + l32;
  const bool row_valid = r < rows_seq;
  if (!row_valid) r = rows_seq - 1;
  const int tok = r / G;
  const int lim = P + tok;                       // last visible position
  const int64_t qrow = (int64_t)(sd.row_off + tok) * a.num_q_heads + g * G + (r - tok * G);
  bf16x8 qreg[KSTEPS][NT];
  {
    const T* qp = reinterpret_cast<const T*>(a.q) + qrow * D;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) load_terms(qp + kk * 16 + hh * 8, qreg[kk]);
  }

  // ---- gather: this wave's page of a tile (K for waves 0..3, V for 4..7), this
  // lane's key and columns in it
  const bool is_v = wave >= 4;
  const char* pool = reinterpret_cast<const char*>(is_v ? a.v_pool : a.k_pool);
  const int page_in_tile = wave & 3;
  const int key16 = lane & 15, quarter = lane >> 4;
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
  auto page_id = [&](int j) __attribute__((always_inline)) {
    const int page = __builtin_amdgcn_readfirstlane(min(j * 4 + page_in_tile, nblk - 1));
    return (uint32_t)bt[page];
  };
  unsigned st[WORDS];
  unsigned char st_scale;
  auto load_tile = [&](int j, uint32_t id) __attribute__((always_inline)) {
    const int page = min(j * 4 + page_in_tile, nblk - 1);
    const int slot = min(key16, L - 1 - page * kBlock);
    const char* p = pool + ((int64_t)min(id, nb_max) * hkv + g) * kPage;
    const char* code = p + slot * (D / 2) + quarter * (D / 8);
    if constexpr (WORDS == 4) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(code);
#pragma unroll
      for (int i = 0; i < 4; ++i) st[i] = w[i];
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2*>(code);
#pragma unroll
      for (int i = 0; i < 2; ++i) st[i] = w[i];
    }
    st_scale = (unsigned char)p[mx_code_bytes(D) + slot * (D / 32) + (D == 128 ? quarter : quarter >> 1)];
  };
  const int st_row = (page_in_tile * 16 + key16) * D, st_swz = swz<D>(key16);
  auto stash = [&](MxHalfTile<D> (&slot)[2]) __attribute__((always_inline)) {
    const float scale = mx_scale(is_v && st_scale == kMxNan ? 0u : st_scale);
    __bf16* to = (is_v ? slot[1].e : slot[0].e) + st_row;
#pragma unroll
    for (int i = 0; i < WORDS; ++i)
      *reinterpret_cast<u32x4*>(to + (((quarter * WORDS + i) ^ st_swz) << 3)) =
          __builtin_bit_cast(u32x4, mx_values(st[i], scale));
  };

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = (f32x16){};
  float m_ref = -INFINITY, l_run = 0.f;
  const float c = a.scale_log2;
  const int g16 = (lane >> 4) & 1;
  const int rsel = (lane & 15) >> 2;
  int koff[KSTEPS], voff[DT][2];
#pragma unroll
  for (int kk = 0; kk < KSTEPS; ++kk) koff[kk] = l32 * D + (((2 * kk + hh) ^ swz<D>(l32)) << 3);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r2 = 0; r2 < 2; ++r2) {
      const int key = 8 * r2 + 4 * hh + rsel;
      const int dcol = dt * 32 + g16 * 16 + 4 * (lane & 3);
      voff[dt][r2] = key * D + (((dcol >> 3) ^ swz<D>(key)) << 3) + (dcol & 7);
    }

  // ---- one tile: scores, mask, online softmax, value product
  auto tile = [&](int j, const MxHalfTile<D> (&slot)[2]) __attribute__((always_inline)) {
    const __bf16* ks = slot[0].e;
    f32x16 s[2] = {(f32x16){}, (f32x16){}};
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(ks + koff[kk] + half * 32 * D));
#pragma unroll
        for (int t = 0; t < NT; ++t)
          s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qreg[kk][t], s[half], 0, 0, 0);
      }
    // element e of half h of a lane's scores is key j*KT + 4*hh + 32h + 8(e/4) + e%4
    if (j * KT + KT - 1 > lim_min) {
      const int thr = lim - j * KT - 4 * hh;
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (half * 32 + 8 * (e >> 2) + (e & 3) > thr) s[half][e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[half][e]);
    const float mxc = pair_max(mx) * c;
    const float m_new = (mxc > m_ref + kRescaleSlack) ? mxc : m_ref;
    const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);
    m_ref = m_new;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
    }
    const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
    const lds_bf16* vl = (const lds_bf16*)slot[1].e;
    float rs[2] = {0.f, 0.f};
#pragma unroll
    for (int kg = 0; kg < 4; ++kg) {
      float pr[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pr[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kg >> 1][(kg & 1) * 8 + e], c, -m_use));
        rs[e & 1] += pr[e];
      }
      bf16x8 pb[NT];
      prob_terms(pr, pb);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(vl + voff[dt][0] + kg * 16 * D));
        const bf16x4 v2 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(vl + voff[dt][1] + kg * 16 * D));
        const bf16x8 vf = __builtin_shufflevector(v1, v2, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int t = 0; t < NT; ++t)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[t], o[dt], 0, 0, 0);
      }
    }
    l_run = l_run * alpha + (rs[0] + rs[1]);
  };

  // ---- main loop.  Step t converts tile t+1, loaded during step t-1, into the
  // other slot, starts loading tile t+2 and computes tile t; the barrier at the
  // end publishes tile t+1 and frees the slot of tile t.  Past the last tile the
  // loads still read pages of the sequence, into a slot no one reads.
  const int n = j1 - j0;
  const bool idle = r0 + wave * 32 >= rows_seq;   // a wave of padding rows only: gathers, no products
  uint32_t id = 0;
  if (n > 0) {
    load_tile(j0, page_id(j0));
    id = page_id(j0 + 1);
    stash(slot0);
    load_tile(j0 + 1, id);
    id = page_id(j0 + 2);
  }
  __syncthreads();
  auto step = [&](int t, const MxHalfTile<D> (&cur)[2], MxHalfTile<D> (&fill)[2]) __attribute__((always_inline)) {
    stash(fill);
    load_tile(j0 + t + 2, id);
    id = page_id(j0 + t + 3);
    if (!idle) tile(j0 + t, cur);
    __syncthreads();
  };
  int t = 0;
  for (; t + 2 <= n; t += 2) {
    step(t, slot0, slot1);
    step(t + 1, slot1, slot0);
  }
  if (t < n) step(t, slot0, slot1);
  if (idle) return;

  // ---- epilogue
  const float l_tot = pair_sum(l_run);
  if (!row_valid) return;
  if (a.direct) {
    const float inv = 1.0f / l_tot;
    T* op = reinterpret_cast<T*>(a.out) + qrow * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        store4(op + dt * 32 + 8 * i + 4 * hh, o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv, o[dt][4 * i + 2] * inv,
               o[dt][4 * i + 3] * inv);
    if (a.lse != nullptr && hh == 0) a.lse[qrow] = (m_ref + __builtin_log2f(l_tot)) * kLn2;
  } else {
    const int64_t set_rows = (int64_t)a.total_rows * a.num_q_heads;
    const int64_t prow = split * set_rows + qrow;
    float* op = a.part_o + prow * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        store4(op + dt * 32 + 8 * i + 4 * hh, o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]);
    if (hh == 0) {
      a.part_ml[prow * 2] = m_ref;
      a.part_ml[prow * 2 + 1] = l_tot;
      // the last split marks the sets that this row tile has no splits for
      for (int x = 1; split == nsplit - 1 && x <= sets - nsplit; ++x) {
        a.part_ml[(prow + x * set_rows) * 2] = -INFINITY;
        a.part_ml[(prow + x * set_rows) * 2 + 1] = -1.f;
      }
    }
  }
}

}  // namespace

hipError_t launch_mx_extend(const ExtendArgs& a, int dtype, int head_dim, int grid, hipStream_t stream) {
  const dim3 g(grid), b(kThreads);
  if (dtype == 0 && head_dim == 128) hipLaunchKernelGGL((mx_extend_kernel<__bf16, 128>), g, b, 0, stream, a);
  else if (dtype == 0 && head_dim == 64) hipLaunchKernelGGL((mx_extend_kernel<__bf16, 64>), g, b, 0, stream, a);
  else if (dtype == 1 && head_dim == 128) hipLaunchKernelGGL((mx_extend_kernel<float, 128>), g, b, 0, stream, a);
  else hipLaunchKernelGGL((mx_extend_kernel<float, 64>), g, b, 0, stream, a);
  return hipGetLastError();
}

}  // namespace kvt
