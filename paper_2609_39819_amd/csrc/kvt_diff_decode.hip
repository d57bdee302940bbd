// Differential attention of one new token per sequence, gfx950.
//
// The formula is kvt_diff.hip's with a suffix of one; the cost is streaming each
// sequence's K/V once from HBM.  Work decomposition, as the decode kernel's:
//   * one workgroup per (sequence, kv-head, key split, up to 16 of the kv-head's
//     query heads), 4 waves; wave w takes the split's 32-key tiles w, w+4, ...,
//     loads one into registers while it computes the one before from its own LDS
//     slot; no barrier in the loop;
//   * a 32-row MFMA block holds both maps of 16 heads: row x is map x/16 of head
//     x%16, its query zero in the other map's columns, so one score product over
//     all D columns serves both maps, and one value product too (half of the
//     score product multiplies zeros, which a stream bound by HBM does not feel);
//   * at the end the four waves' (m, l, O) merge through LDS; the merged row is
//     either turned into the output there (difference of the maps, norm) or a
//     partial of its key split.
// bf16 storage hands the value product each probability as two bf16 numbers, as the
// extend kernel's and for its reason; beside a stream bound by HBM the
// second product costs at most 1.5 % of a step (64 contexts of 1024..16384 keys,
// heads of 128, 247.4 -> 248.5 us, of 64 124.1 -> 126.0).  fp32 storage runs fp32
// matrix products throughout; at 25 GB/s a workgroup they bound it (5.4 TB/s on a
// full chip, bf16 6.7).
#include <type_traits>

#include "kvt_diff_device.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kWaves = kDecWaves;
constexpr int kTK = kDecKeysPerTile;   // keys per tile = 2 pages

// One wave's slot: its K tile then its V tile, [key][D] as stored, with the
// 16-byte chunks of each key row XOR-swizzled; later its O rows, [row][D] fp32.
template <typename T, int D>
struct DecSlot {
  T k[kTK * D];
  T v[kTK * D];
};

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) * D > 256 ? 1 : 2) void diff_decode_kernel(const DiffArgs a) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int ROWB = D * (int)sizeof(T);       // bytes per key row
  constexpr int CHUNKS = ROWB / 16;
  constexpr int RPR = 1024 / ROWB;               // key rows per 1 KiB wave load
  constexpr int NLD = kTK * ROWB / 1024;         // 1 KiB loads per tensor per tile
  constexpr int DT = D / 32;
  constexpr int KF = kBf16 ? D / 16 : D / 8;     // query fragments
  constexpr float kRescaleSlack = 8.0f;
  __shared__ __attribute__((aligned(1024))) DecSlot<T, D> ring[kWaves];
  __shared__ float ml[kWaves][32][2];            // per wave and row: m (log2 units), l

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5;
  const int l32 = lane & 31;
  // chunk swizzles of K and V rows, as the extend kernel's
  auto swizzle_k = [](int key) __attribute__((always_inline)) {
    if constexpr (kBf16) return swz<D>(key);
    else return key & 15;
  };
  auto swizzle_v = [](int key) __attribute__((always_inline)) {
    if constexpr (kBf16) return swz<D>(key);
    else return (key & 4) << 1;
  };

  // ---- which (sequence, kv-head, key split, head chunk) this workgroup owns
  const int hkv = a.num_kv_heads;
  const int G = a.group;
  const int chunks = (G + kDiffDecHeads - 1) / kDiffDecHeads;
  const int g = blockIdx.x % hkv;
  const int rest = blockIdx.x / hkv;
  const int unit = rest / chunks;
  const int head0 = (rest - unit * chunks) * kDiffDecHeads;   // first of this workgroup's heads in the group
  const int heads = min(kDiffDecHeads, G - head0);
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const SeqDesc sd = a.seq[si];
  const int nsplit = a.nsplit[si];
  const int split = unit - a.unit_begin[si];
  const int L = sd.prefix + 1;                   // keys 0..P_b
  const int nblk = (L + kBlock - 1) / kBlock;
  const int ntk = (L + kTK - 1) / kTK;
  const int per_split = (ntk + nsplit - 1) / nsplit;
  const int j0 = split * per_split;
  const int j1 = min(ntk, j0 + per_split);
  const int nt = j1 - j0 > wave ? (j1 - j0 - wave + kWaves - 1) / kWaves : 0;   // this wave's tiles

  // ---- this lane's query row: map l32/16 of head l32%16 (heads past the last
  // repeat it and are dropped), zero in the other map's columns
  const int64_t first_row = (int64_t)sd.row_off * a.num_q_heads + g * G + head0;
  typedef typename std::conditional<kBf16, bf16x8, f32x4>::type QFrag;
  QFrag qreg[KF];
  {
    const T* qp = reinterpret_cast<const T*>(a.q) + (first_row + min(l32 & 15, heads - 1)) * D;
#pragma unroll
    for (int kk = 0; kk < KF; ++kk) {
      const bool mine = (kk >= KF / 2) == (l32 >= 16);
      QFrag f;
      if constexpr (kBf16) f = __builtin_bit_cast(bf16x8, load8(qp + kk * 16 + hh * 8));
      else f = load4(qp + kk * 8 + hh * 4);
      qreg[kk] = mine ? f : (QFrag){};
    }
  }

  const T* kpool = reinterpret_cast<const T*>(a.k_pool);
  const T* vpool = reinterpret_cast<const T*>(a.v_pool);
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;

  // ---- gather geometry: load i of a tile covers key rows RPR*i .. RPR*i+RPR-1
  // (all in one page); lane l lands at byte 16*l of that 1 KiB run, i.e. row
  // RPR*i + l/CHUNKS, physical chunk l%CHUNKS, logical chunk
  // (l%CHUNKS) ^ swizzle(row)
  auto page_ids = [&](int j, uint32_t (&ids)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = __builtin_amdgcn_readfirstlane(min(j * 2 + p, nblk - 1));
      const uint32_t raw = (uint32_t)bt[page];
      ids[p] = __builtin_amdgcn_readfirstlane(raw > nb_max ? nb_max : raw);
    }
  };
  struct Stage {
    u32x4 k[NLD], v[NLD];
  };
  // positions past the end read the last real position (finite; weight 0);
  // each page is read once: nontemporal loads
  auto load_tile = [&](int j, const uint32_t (&ids)[2], Stage& st) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int p = (RPR * i) / kBlock;
      const int page = min(j * 2 + p, nblk - 1);
      const int key = RPR * i + lane / CHUNKS;
      const int slot = min(key & (kBlock - 1), L - 1 - page * kBlock);
      const int64_t off = ((((int64_t)ids[p] * hkv + g) << 4) + slot) * D;
      constexpr int PER = 16 / (int)sizeof(T);
      const T* ks = kpool + off + ((lane % CHUNKS) ^ swizzle_k(key)) * PER;
      const T* vs = vpool + off + ((lane % CHUNKS) ^ swizzle_v(key)) * PER;
      st.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(ks));
      st.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vs));
    }
  };
  // (and their values become 0: the last real one may be an infinity, which
  // its own weight takes in once)
  auto stash = [&](int j, Stage& st, DecSlot<T, D>& dst) __attribute__((always_inline)) {
    if ((j + 1) * kTK > L) {
#pragma unroll
      for (int i = 0; i < NLD; ++i)
        if (j * kTK + RPR * i + lane / CHUNKS >= L) st.v[i] = (u32x4){0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      reinterpret_cast<u32x4*>(dst.k)[i * 64 + lane] = st.k[i];
      reinterpret_cast<u32x4*>(dst.v)[i * 64 + lane] = st.v[i];
    }
  };

  f32x16 o[DT];
  float m_ref, l_run;
  const float c = a.scale_log2;
  const int g16 = (lane >> 4) & 1;
  const int rsel = (lane & 15) >> 2;

  // ---- one 32-key tile starting at key kb: scores, softmax, value product
  auto tile = [&](const DecSlot<T, D>& sl, int kb) __attribute__((always_inline)) {
    f32x16 s = (f32x16){};
#pragma unroll
    for (int kk = 0; kk < KF; ++kk) {
      const u32x4 kf = reinterpret_cast<const u32x4*>(sl.k)[l32 * CHUNKS + ((2 * kk + hh) ^ swizzle_k(l32))];
      if constexpr (kBf16) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), qreg[kk], s, 0, 0, 0);
      } else {
        const f32x4 k4 = __builtin_bit_cast(f32x4, kf);
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k4[i], qreg[kk][i], s, 0, 0, 0);
      }
    }
    if (kb + kTK > L) {   // the sequence ends inside this tile
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (kb + 8 * (e >> 2) + 4 * hh + (e & 3) >= L) s[e] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    const float mxc = pair_max(mx) * c;
    const float m_new = (mxc > m_ref + kRescaleSlack) ? mxc : m_ref;
    const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);
    m_ref = m_new;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
    }
    const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
    float rs = 0.f;
    if constexpr (kBf16) {
      const lds_bf16* vl = (const lds_bf16*)sl.v;
#pragma unroll
      for (int kg = 0; kg < 2; ++kg) {
        u32x4 wv, lv;
#pragma unroll
        for (int q2 = 0; q2 < 4; ++q2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kg * 8 + 2 * q2], c, -m_use));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kg * 8 + 2 * q2 + 1], c, -m_use));
          unsigned w, rest;
          two_numbers(p0, p1, w, rest);
          wv[q2] = w;
          lv[q2] = rest;
          rs += p0 + p1;
        }
        const bf16x8 pb = __builtin_bit_cast(bf16x8, wv), pl = __builtin_bit_cast(bf16x8, lv);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          bf16x4 v[2];
#pragma unroll
          for (int r2 = 0; r2 < 2; ++r2) {
            const int key = 8 * r2 + 4 * hh + rsel;
            const int dcol = dt * 32 + g16 * 16 + 4 * (lane & 3);
            const int off = key * D + (((dcol >> 3) ^ swizzle_v(key)) << 3) + (dcol & 7);
            v[r2] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(vl + off + kg * 16 * D));
          }
          const bf16x8 vf = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb, o[dt], 0, 0, 0);
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pl, o[dt], 0, 0, 0);
        }
      }
    } else {
      // product e takes keys 8 (e/4) + e%4 and the fourth after it, one per lane half
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -m_use));
        rs += p;
        const int key = 8 * (e >> 2) + 4 * hh + (e & 3);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const int col = dt * 32 + l32;
          const float vf = sl.v[key * D + (((col >> 2) ^ swizzle_v(key)) << 2) + (col & 3)];
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, p, o[dt], 0, 0, 0);
        }
      }
    }
    l_run = l_run * alpha + rs;
  };

  // ---- this wave's tiles j0 + wave + kWaves*i.  Step i stores tile i, which
  // its loads brought into registers, into the slot, starts loading tile i+1
  // and computes tile i (the wave's LDS operations run in order, so the
  // stores follow the reads of the tile before).
  DecSlot<T, D>& mine = ring[wave];
  auto jt = [&](int i) { return j0 + wave + kWaves * i; };
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = (f32x16){};
  m_ref = -INFINITY, l_run = 0.f;
  Stage st;
  uint32_t ids[2];
  if (nt > 0) {
    page_ids(jt(0), ids);
    load_tile(jt(0), ids, st);
    page_ids(jt(1), ids);
  }
  for (int i = 0; i < nt; ++i) {
    stash(jt(i), st, mine);
    if (i + 1 < nt) {
      load_tile(jt(i + 1), ids, st);
      page_ids(jt(i + 2), ids);
    }
    tile(mine, jt(i) * kTK);
  }

  // ---- merge the four waves.  Each wave parks its O rows in its own slot (its
  // loads have landed and its reads of the slot precede these writes in LDS
  // order), four columns a piece, the pieces of a row XOR-swizzled by the row.
  static_assert(sizeof(DecSlot<T, D>) >= 32 * D * sizeof(float), "merge buffer");
  constexpr int Q4 = D / 4;
  const float l_tot = pair_sum(l_run) * (kBf16 ? kOver : 1.0f);
  f32x4* ow = reinterpret_cast<f32x4*>(&mine);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      ow[l32 * Q4 + ((dt * 8 + 2 * i + hh) ^ (l32 & (Q4 - 1)))] =
          (f32x4){o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
  if (hh == 0) {
    ml[wave][l32][0] = m_ref;
    ml[wave][l32][1] = l_tot;
  }
  __syncthreads();
  // Q4 lanes per head, four columns each
  constexpr int PER = kWaves * 64 / Q4;          // heads at a time
  const int lq = tid % Q4;
  for (int h0 = 0; h0 < heads; h0 += PER) {
    const int hd = h0 + tid / Q4;
    const bool live = hd < heads;
    const int hs = live ? hd : heads - 1;
    float top[2], sum[2] = {0.f, 0.f};
    f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int row = 16 * m + hs;
      top[m] = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top[m] = fmaxf(top[m], ml[w][row][0]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = ml[w][row][0];
        const float wt = (mw == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(mw - top[m]);
        sum[m] += wt * ml[w][row][1];
        acc[m] += wt * reinterpret_cast<const f32x4*>(&ring[w])[row * Q4 + (lq ^ (row & (Q4 - 1)))];
      }
    }
    const int64_t row = first_row + hs;
    if (nsplit == 1) {
      const float lam = a.lambda[(int64_t)sd.row_off * a.lambda_stride + g * G + head0 + hs];
      const float inv0 = 1.0f / sum[0], inv1 = 1.0f / sum[1];
      f32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = map_difference(acc[0][i], inv0, acc[1][i], inv1, lam);
      float scale = a.out_scale;
      f32x4 w = {1.f, 1.f, 1.f, 1.f};
      if (a.norm_weight != nullptr) {
        float sq = y[0] * y[0] + y[1] * y[1] + y[2] * y[2] + y[3] * y[3];
#pragma unroll
        for (int d = Q4 / 2; d > 0; d >>= 1) sq += __shfl_xor(sq, d);
        scale *= 1.0f / __builtin_sqrtf(sq * (1.0f / D) + a.eps);
        w = load4(a.norm_weight + lq * 4);
      }
      y *= scale;
      if (live)
        store4(reinterpret_cast<T*>(a.out) + row * D + lq * 4, y[0] * w[0], y[1] * w[1], y[2] * w[2], y[3] * w[3]);
    } else if (live) {
      const int64_t prow = a.part_row[si] + (int64_t)split * a.num_q_heads + g * G + head0 + hs;
#pragma unroll
      for (int m = 0; m < 2; ++m) *reinterpret_cast<f32x4*>(a.part_o + (prow * 2 + m) * D + lq * 4) = acc[m];
      if (lq == 0) *reinterpret_cast<f32x4*>(a.part_ml + prow * 4) = (f32x4){top[0], sum[0], top[1], sum[1]};
    }
  }
}

// One workgroup per CU is asked for by LDS that the kernel does not use: more
// than half of a CU's 160 KB in all.
template <typename T, int D>
void launch_as(const DiffArgs& a, dim3 grid, bool one_per_cu, hipStream_t stream) {
  constexpr unsigned kUsed = kWaves * sizeof(DecSlot<T, D>), kAlone = 84 * 1024;
  hipLaunchKernelGGL((diff_decode_kernel<T, D>), grid, dim3(kWaves * 64),
                     one_per_cu && kAlone > kUsed ? kAlone - kUsed : 0, stream, a);
}

}  // namespace

hipError_t launch_diff_decode(const DiffArgs& a, int dtype, int head_dim, int grid, bool one_per_cu,
                              hipStream_t stream) {
  const dim3 g(grid);
  if (dtype == 0 && head_dim == 128) launch_as<__bf16, 128>(a, g, one_per_cu, stream);
  else if (dtype == 0 && head_dim == 64) launch_as<__bf16, 64>(a, g, one_per_cu, stream);
  else if (dtype == 1 && head_dim == 128) launch_as<float, 128>(a, g, one_per_cu, stream);
  else launch_as<float, 64>(a, g, one_per_cu, stream);
  return hipGetLastError();
}

}  // namespace kvt
