// Differential attention over a paged KV cache, gfx950: a chunk of new tokens.
//
// A head's columns hold two maps of d = D/2 columns.  With K_b[j] the cached
// keys, V_b[j] the cached values and j running over the visible positions,
//   A_m = softmax_j(scale * <q_m, K_b[j]_m>),   m = 0, 1,
//   y = sum_j (A_0[j] - lambda * A_1[j]) V_b[j],
//   out = out_scale * w * y / sqrt(mean(y^2) + eps)      (w given), else out_scale * y.
// The sums of both softmaxes are known only after the last key, so one pass
// over the keys keeps an output per map: 2 D flops per (head, key) for the
// scores and 2 x 2 D for the values.
//
// Work decomposition: one workgroup per (sequence, kv-head, 128 packed query
// rows, key split), as the extend kernel's (row r = token r/G, head g*G + r%G);
// 4 waves of 32 rows.  A wave computes both maps of its rows, so each V fragment
// read from LDS feeds the products of both, and one map's products run beside
// the other's exponentials.  S^T = K Q^T (keys on the MFMA rows, queries on the
// columns), so a query's scores sit in one lane pair (l, l+32) and leave the
// accumulators in the layout that the value product takes them in.
//
// bf16 storage: v_mfma_f32_32x32x16_bf16, tiles of 64 keys, probabilities
// rounded to bf16 for the value product (their sum adds the rounded ones).
// fp32 storage: v_mfma_f32_32x32x2_f32, tiles of 32 keys, nothing rounded: the
// difference of two maps has the error of the larger one, so what bf16 inputs
// lose anyway fp32 ones would lose here.
//
// Masked positions.  Their scores are replaced by -inf, so their weight is
// exactly 0 whatever K holds; positions past the end of the sequence and unused
// page slots read the last real position instead.  But the value product
// multiplies V by that 0, and a visible position of one row is a masked one of
// another: in the tiles that reach past some row's limit a non-finite value is
// looked for first, and if there is one it is added to the rows that see it by
// hand and replaced by 0 for the product.
#include <type_traits>

#include "kvt_device.h"
#include "kvt_internal.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kThreads = kDiffWaves * 64;

// Shapes of one storage type and head width.  Tiles are [key][D] in LDS as
// stored, the 16-byte chunks of each key row XOR-swizzled.
template <typename T, int D>
struct Shape {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int KT = kBf16 ? 64 : 32;            // keys per tile
  static constexpr int HALVES = KT / 32;                // 32-key MFMA blocks per tile
  static constexpr int ROWB = D * (int)sizeof(T);       // bytes per key row
  static constexpr int CHUNKS = ROWB / 16;
  static constexpr int RPR = 1024 / ROWB;               // key rows per 1 KiB wave load
  static constexpr int DT = D / 32;                     // 32-wide output column tiles
  // bf16: swz (kvt_device.h).  fp32: a row is a whole number of 256-byte bank
  // cycles, and 16 keys read the same chunk column at once.
  static __device__ __forceinline__ int swizzle(int key) {
    if constexpr (kBf16) return swz<D>(key);
    else return key & 15;
  }
};

// Whether a word of stored values holds an infinity or a NaN, and the word with 0 in their place.
template <typename T>
__device__ __forceinline__ bool non_finite(unsigned w) {
  if constexpr (sizeof(T) == 2) return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
  else return (w & 0x7f800000u) == 0x7f800000u;
}
template <typename T>
__device__ __forceinline__ unsigned finite_part(unsigned w) {
  if constexpr (sizeof(T) == 2)
    return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
  else return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
}

// One K or V tile; a ring slot is one object holding K then V.
template <typename T, int D>
struct HalfTile {
  T e[Shape<T, D>::KT * D];
};
template <typename T, int D>
struct Slot {
  HalfTile<T, D>& k;
  HalfTile<T, D>& v;
};

// A wave's query rows as the B operand of the score product, a map's half of
// the columns after the other's.  bf16: fragment kk holds columns 16 kk + 8 hh
// .. + 7.  fp32: element i of chunk pair kk is column 8 kk + 4 hh + i.
template <typename T, int D>
struct Queries;
template <int D>
struct Queries<__bf16, D> {
  bf16x8 f[D / 16];
  __device__ __forceinline__ void load(const __bf16* p, int hh) {
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) f[kk] = __builtin_bit_cast(bf16x8, load8(p + kk * 16 + hh * 8));
  }
};
template <int D>
struct Queries<float, D> {
  f32x4 f[D / 8];
  __device__ __forceinline__ void load(const float* p, int hh) {
#pragma unroll
    for (int kk = 0; kk < D / 8; ++kk) f[kk] = *reinterpret_cast<const f32x4*>(p + kk * 8 + hh * 4);
  }
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 1) void diff_extend_kernel(const DiffArgs a) {
  using S = Shape<T, D>;
  constexpr int KT = S::KT, HALVES = S::HALVES, DT = S::DT, RPR = S::RPR;
  constexpr int PAGES = KT / kBlock;                              // pages per tile
  constexpr int NREG = KT * S::ROWB / 1024 / kDiffWaves;          // 1 KiB loads per wave per tensor
  constexpr float kRescaleSlack = 8.0f;                           // log2 headroom before O is rescaled
  typedef typename std::conditional<S::kBf16, bf16x8, f32x16>::type Probs;
  constexpr int NP = S::kBf16 ? KT / 16 : HALVES;                 // probability operands per map
  __shared__ __attribute__((aligned(1024))) HalfTile<T, D> slot0[2];   // K, V
  __shared__ __attribute__((aligned(1024))) HalfTile<T, D> slot1[2];
  const Slot<T, D> tile0{slot0[0], slot0[1]}, tile1{slot1[0], slot1[1]};

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5;     // lane half
  const int l32 = lane & 31;

  // ---- which (sequence, kv-head, row tile, key split) this workgroup owns
  const int hkv = a.num_kv_heads;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const SeqDesc sd = a.seq[si];
  const int nsplit = a.nsplit[si];
  const int local = unit - a.unit_begin[si];
  const int G = a.group;
  const int rows_seq = sd.suffix * G;
  const int ntile = (rows_seq + kDiffTileRows - 1) / kDiffTileRows;
  const int rt = ntile - 1 - local / nsplit;   // longest (last) row tile first
  const int split = local % nsplit;
  const int r0 = rt * kDiffTileRows;
  const int P = sd.prefix;
  const int L = P + sd.suffix;                 // positions that can be read
  const int nblk = (L + kBlock - 1) / kBlock;

  // keys up to the tile's last query's own position, evenly over the splits
  const int t_last = min(sd.suffix - 1, (r0 + kDiffTileRows - 1) / G);
  const int ntiles_kv = (P + t_last + KT) / KT;
  const int per_split = (ntiles_kv + nsplit - 1) / nsplit;
  const int j0 = split * per_split;
  const int j1 = min(ntiles_kv, j0 + per_split);
  const int lim_min = P + r0 / G;              // smallest last-visible key of the tile

  // ---- this lane's query row
  int r = r0 + wave * 32 + l32;
  const bool row_valid = r < rows_seq;
  if (!row_valid) r = rows_seq - 1;
  const int t_row = r / G;
  const int h_row = g * G + (r - t_row * G);
  const int lim = P + t_row;                   // last visible position
  const int64_t qrow = (int64_t)(sd.row_off + t_row) * a.num_q_heads + h_row;
  Queries<T, D> q;
  q.load(reinterpret_cast<const T*>(a.q) + qrow * D, hh);

  const char* kpool = reinterpret_cast<const char*>(a.k_pool);
  const char* vpool = reinterpret_cast<const char*>(a.v_pool);
  // read-only here: a constant-address-space view lets wave-uniform page
  // lookups become scalar loads
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;

  // ---- gather geometry: wave w, load i covers key rows RPR*(w + 4i) ..
  // +RPR-1 of the tile, all inside one page.  Lane l lands at LDS byte 16*l of
  // that 1 KiB run, i.e. row RPR*(w + 4i) + l/CHUNKS, physical chunk l%CHUNKS,
  // so it fetches logical chunk (l%CHUNKS) ^ swizzle(row).
  constexpr uint32_t ROWM = S::ROWB - 1;
  int lds_off[NREG], page_in_tile[NREG];
  uint32_t lane_off[NREG];                     // this lane's byte offset within its page run
#pragma unroll
  for (int i = 0; i < NREG; ++i) {
    const int run = wave + kDiffWaves * i;
    const int keyrow = RPR * run + lane / S::CHUNKS;
    page_in_tile[i] = (RPR * run) / kBlock;
    lds_off[i] = run * 1024;                   // bytes
    lane_off[i] = (uint32_t)((keyrow & (kBlock - 1)) * S::ROWB + (((lane % S::CHUNKS) ^ S::swizzle(keyrow)) << 4));
  }
  // page ids as the block table has them, clamped into the pool where they are used
  auto page_ids = [&](int jn, uint32_t (&ids)[NREG]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NREG; ++i) {
      const int page = __builtin_amdgcn_readfirstlane(min(jn * PAGES + page_in_tile[i], nblk - 1));
      ids[i] = (uint32_t)bt[page];
    }
  };
  // positions past the end of the sequence take the last real position's offset
  const uint32_t tail = (uint32_t)((L - 1) & (kBlock - 1)) * (ROWM + 1);
  auto gather = [&](int jn, const uint32_t (&ids)[NREG], const Slot<T, D>& dst) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NREG; ++i) {
      const uint32_t last = jn * PAGES + page_in_tile[i] >= nblk - 1 ? tail : (kBlock - 1) * (ROWM + 1);
      const uint32_t lb = min(lane_off[i], last | (lane_off[i] & ROWM));
      const int64_t base = (((int64_t)min(ids[i], nb_max) * hkv + g) << 4) * S::ROWB;
      __builtin_amdgcn_global_load_lds((const void*)(kpool + base + lb),
                                       (__attribute__((address_space(3))) void*)((lds_char*)dst.k.e + lds_off[i]), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const void*)(vpool + base + lb),
                                       (__attribute__((address_space(3))) void*)((lds_char*)dst.v.e + lds_off[i]), 16, 0, 0);
    }
  };

  f32x16 o[2][DT];
  float m_ref[2], l_run[2];   // reference max of scale*log2e*score; this lane's share of sum 2^(s*c - m_ref)
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    m_ref[m] = -INFINITY, l_run[m] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[m][dt] = (f32x16){};
  }
  const float c = a.scale_log2;

  // ---- S^T = K Q^T of one tile and map
  auto scores = [&](const Slot<T, D>& tl, int m, f32x16 (&s)[HALVES]) __attribute__((always_inline)) {
#pragma unroll
    for (int half = 0; half < HALVES; ++half) s[half] = (f32x16){};
    if constexpr (S::kBf16) {
#pragma unroll
      for (int k0 = 0; k0 < D / 32; ++k0) {
        const int kk = m * (D / 32) + k0;
        const int off = l32 * D + (((2 * kk + hh) ^ S::swizzle(l32)) << 3);
#pragma unroll
        for (int half = 0; half < HALVES; ++half) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(tl.k.e + off + half * 32 * D));
          s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q.f[kk], s[half], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int k0 = 0; k0 < D / 16; ++k0) {
        const int kk = m * (D / 16) + k0;
        const int off = l32 * D + (((2 * kk + hh) ^ S::swizzle(l32)) << 2);
        const f32x4 kf = *reinterpret_cast<const f32x4*>(tl.k.e + off);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[i], q.f[kk][i], s[0], 0, 0, 0);
      }
    }
  };
  // ---- causal mask, row max and the reference-max update of one map.  Element
  // e of block `half` is key j*KT + 32 half + 8 (e/4) + 4 hh + e%4.  The reference
  // only moves when a tile max passes it by more than the slack; O and l are then
  // rescaled (rare after the first tiles).
  auto settle = [&](int j, int m, f32x16 (&s)[HALVES]) __attribute__((always_inline)) {
    if (j * KT + KT - 1 > lim_min) {
      const int thr = lim - j * KT - 4 * hh;
#pragma unroll
      for (int half = 0; half < HALVES; ++half)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (half * 32 + 8 * (e >> 2) + (e & 3) > thr) s[half][e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int half = 0; half < HALVES; ++half)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[half][e]);
    const float mxc = pair_max(mx) * c;
    const float m_new = (mxc > m_ref[m] + kRescaleSlack) ? mxc : m_ref[m];
    // 1 when unchanged, 0 when leaving -inf; kept at 1 while the row has seen no visible key
    const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m_ref[m] - m_new);
    m_ref[m] = m_new;
    l_run[m] *= alpha;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[m][dt] *= alpha;
    }
  };
  // ---- probabilities of a settled tile as the B operands of the value product
  auto probs = [&](int m, const f32x16 (&s)[HALVES], Probs (&pb)[NP]) __attribute__((always_inline)) {
    const float m_use = (m_ref[m] == -INFINITY) ? 0.f : m_ref[m];
    float rs = 0.f;
    if constexpr (S::kBf16) {
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int kg = 0; kg < NP; ++kg) {
        const int half = kg >> 1, b0 = (kg & 1) * 8;
        u32x4 wv;
#pragma unroll
        for (int q2 = 0; q2 < 4; ++q2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[half][b0 + 2 * q2], c, -m_use));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[half][b0 + 2 * q2 + 1], c, -m_use));
          const bf16x2 pp = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
          rs = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, rs, false);
          wv[q2] = __builtin_bit_cast(unsigned, pp);
        }
        pb[kg] = __builtin_bit_cast(bf16x8, wv);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        pb[0][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][e], c, -m_use));
        rs += pb[0][e];
      }
    }
    l_run[m] += rs;
  };
  // ---- O^T += V^T P^T of both maps, each V fragment feeding two products
  const int g16 = (lane >> 4) & 1, rsel = (lane & 15) >> 2;
  auto values = [&](const Slot<T, D>& tl, const Probs (&pb)[2][NP]) __attribute__((always_inline)) {
    if constexpr (S::kBf16) {
      const lds_bf16* vl = (const lds_bf16*)tl.v.e;
#pragma unroll
      for (int kg = 0; kg < NP; ++kg)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          bf16x4 v[2];
#pragma unroll
          for (int r2 = 0; r2 < 2; ++r2) {
            const int key = 8 * r2 + 4 * hh + rsel;          // key within a 16-key group
            const int dcol = dt * 32 + g16 * 16 + 4 * (lane & 3);
            const int off = key * D + (((dcol >> 3) ^ S::swizzle(key)) << 3) + (dcol & 7);
            v[r2] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(vl + off + kg * 16 * D));
          }
          const bf16x8 vf = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int m = 0; m < 2; ++m) o[m][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[m][kg], o[m][dt], 0, 0, 0);
        }
    } else {
      // product e takes keys 8 (e/4) + e%4 and the fourth after it, one per lane half
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 8 * (e >> 2) + 4 * hh + (e & 3);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const int col = dt * 32 + l32;
          const float vf = tl.v.e[key * D + (((col >> 2) ^ S::swizzle(key)) << 2) + (col & 3)];
#pragma unroll
          for (int m = 0; m < 2; ++m) o[m][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, pb[m][0][e], o[m][dt], 0, 0, 0);
        }
      }
    }
  };

  // ---- non-finite values in a tile with masked positions (see the top): whether
  // there is one (workgroup-uniform), ...
  constexpr int VCHUNKS = KT * S::ROWB / 16 / kThreads;   // 16-byte pieces of a V tile per thread
  auto odd_values = [&](int j, const Slot<T, D>& tl) __attribute__((always_inline)) {
    if (j * KT + KT - 1 <= lim_min) return false;
    const u32x4* p = reinterpret_cast<const u32x4*>(tl.v.e);
    bool odd = false;
#pragma unroll
    for (int i = 0; i < VCHUNKS; ++i) {
      const u32x4 w = p[tid + kThreads * i];
#pragma unroll
      for (int x = 0; x < 4; ++x) odd = odd || non_finite<T>(w[x]);
    }
    return __syncthreads_or(odd) != 0;
  };
  // ... its part in the rows that see it, ...
  auto add_odd = [&](int j, const Slot<T, D>& tl) __attribute__((always_inline)) {
    const unsigned* words = reinterpret_cast<const unsigned*>(tl.v.e);
    constexpr int WORDS = S::ROWB / 4;
    for (int key = 0; key < KT; ++key) {
      bool odd = false;
      for (int w = lane; w < WORDS; w += 64) odd = odd || non_finite<T>(words[key * WORDS + w]);
      if (__builtin_amdgcn_ballot_w64(odd) == 0) continue;
      const bool seen = j * KT + key <= lim;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          constexpr int PER = 16 / (int)sizeof(T);
          const int d = dt * 32 + 8 * (e >> 2) + 4 * hh + (e & 3);
          const float v = (float)tl.v.e[key * D + ((d / PER) ^ S::swizzle(key)) * PER + d % PER];
          if (seen && !__builtin_isfinite(v))
#pragma unroll
            for (int m = 0; m < 2; ++m) o[m][dt][e] += v;
        }
    }
  };
  // ... and its removal from the tile
  auto clear_odd = [&](const Slot<T, D>& tl) __attribute__((always_inline)) {
    u32x4* p = reinterpret_cast<u32x4*>(tl.v.e);
#pragma unroll
    for (int i = 0; i < VCHUNKS; ++i) {
      u32x4 w = p[tid + kThreads * i];
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = finite_part<T>(w[x]);
      p[tid + kThreads * i] = w;
    }
  };

  // ---- main loop: step t computes tile t while tile t+1 streams into the other
  // slot (past the last tile the gather still reads clamped, in-bounds pages
  // into a slot no one reads); the wait + barrier publishes tile t+1 and frees
  // the slot of tile t.
  const int n = j1 - j0;
  uint32_t ids[NREG];
  page_ids(j0, ids);
  if (n > 0) gather(j0, ids, tile0);
  page_ids(j0 + 1, ids);
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  __syncthreads();
  const bool idle = r0 + wave * 32 >= rows_seq;   // a wave past the last row only takes part in the gather
  auto step = [&](int t, const Slot<T, D>& cur, const Slot<T, D>& fill) __attribute__((always_inline)) {
    gather(j0 + t + 1, ids, fill);
    page_ids(j0 + t + 2, ids);
    const bool odd = odd_values(j0 + t, cur);
    f32x16 s[2][HALVES];
    Probs pb[2][NP];
    if (!idle) {
#pragma unroll
      for (int m = 0; m < 2; ++m) scores(cur, m, s[m]);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        settle(j0 + t, m, s[m]);
        probs(m, s[m], pb[m]);
      }
    }
    if (odd) {
      if (!idle) add_odd(j0 + t, cur);
      __syncthreads();
      clear_odd(cur);
      __syncthreads();
    }
    if (!idle) values(cur, pb);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __syncthreads();
  };
  for (int t = 0; t < n; t += 2) {
    step(t, tile0, tile1);
    if (t + 1 >= n) break;
    step(t + 1, tile1, tile0);
  }

  // ---- epilogue
  float l_tot[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) l_tot[m] = pair_sum(l_run[m]);
  if (nsplit == 1) {
    const float lam = a.lambda[(int64_t)(sd.row_off + t_row) * a.lambda_stride + h_row];
    const float inv0 = 1.0f / l_tot[0], inv1 = 1.0f / l_tot[1];
    float sq = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float y = map_difference(o[0][dt][e], inv0, o[1][dt][e], inv1, lam);
        o[0][dt][e] = y;
        sq += y * y;
      }
    sq = pair_sum(sq);
    if (!row_valid) return;
    float scale = a.out_scale;
    if (a.norm_weight != nullptr) scale *= 1.0f / __builtin_sqrtf(sq * (1.0f / D) + a.eps);
    T* op = reinterpret_cast<T*>(a.out) + qrow * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = dt * 32 + 8 * i + 4 * hh;
        f32x4 w = {1.f, 1.f, 1.f, 1.f};
        if (a.norm_weight != nullptr) w = load4(a.norm_weight + d);
        store4(op + d, o[0][dt][4 * i] * scale * w[0], o[0][dt][4 * i + 1] * scale * w[1],
               o[0][dt][4 * i + 2] * scale * w[2], o[0][dt][4 * i + 3] * scale * w[3]);
      }
  } else {
    if (!row_valid) return;
    const int64_t rows = (int64_t)sd.suffix * a.num_q_heads;
    const int64_t prow = a.part_row[si] + split * rows + (int64_t)t_row * a.num_q_heads + h_row;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float* op = a.part_o + (prow * 2 + m) * D;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = dt * 32 + 8 * i + 4 * hh;
          store4(op + d, o[m][dt][4 * i], o[m][dt][4 * i + 1], o[m][dt][4 * i + 2], o[m][dt][4 * i + 3]);
        }
    }
    if (hh == 0)
      *reinterpret_cast<f32x4*>(a.part_ml + prow * 4) = (f32x4){m_ref[0], l_tot[0], m_ref[1], l_tot[1]};
  }
}

// Joins the key splits of each row (fixed order): with m* = max_s m_s and
// w_s = 2^(m_s - m*), map m is sum_s w_s O_s / sum_s w_s l_s; then the maps'
// difference and its norm as in the kernel's own epilogue.  D/4 lanes per row,
// four columns each; the weights of the splits are formed once per row, one
// split per lane, and shared through LDS.  Every split is multiplied by its
// weight, be it 0, so an infinity or a NaN among the values gives the unsplit
// call's.  args: the sequences with more than one split; unit_begin counts
// their rows.
constexpr int kAhead = 8;   // splits whose pieces are in flight at once

template <typename T, int D>
__global__ __launch_bounds__(256) void diff_combine_kernel(const DiffArgs a) {
  constexpr int Q4 = D / 4, ROWS = 256 / Q4;       // lanes per row, rows per workgroup
  constexpr int PER = (kMaxPartials + Q4 - 1) / Q4;
  __shared__ float wts[ROWS][2][kMaxPartials];
  const int lr = threadIdx.x / Q4, lq = threadIdx.x % Q4;
  const int total = a.unit_begin[a.nseq];
  const int idx = blockIdx.x * ROWS + lr;
  const bool live = idx < total;
  const int row = live ? idx : total - 1;
  const int si = find_seq(a.unit_begin, a.nseq, row);
  const SeqDesc sd = a.seq[si];
  const int nsplit = a.nsplit[si];
  const int local = row - a.unit_begin[si];        // token * Hq + head within the sequence
  const int64_t rows = (int64_t)sd.suffix * a.num_q_heads;
  const int64_t first = a.part_row[si] + (int64_t)local;

  float m[2][PER], l[2][PER], top[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int s = lq + k * Q4;
    f32x4 e = {-INFINITY, 0.f, -INFINITY, 0.f};
    if (s < nsplit) e = load4(a.part_ml + (first + s * rows) * 4);
#pragma unroll
    for (int x = 0; x < 2; ++x) m[x][k] = e[2 * x], l[x][k] = e[2 * x + 1], top[x] = fmaxf(top[x], e[2 * x]);
  }
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int d = Q4 / 2; d > 0; d >>= 1) top[x] = fmaxf(top[x], __shfl_xor(top[x], d));
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int x = 0; x < 2; ++x) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int s = lq + k * Q4;
      const float w = (m[x][k] == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m[x][k] - top[x]);
      sum[x] += w * l[x][k];
      if (s < nsplit) wts[lr][x][s] = w;
    }
#pragma unroll
    for (int d = Q4 / 2; d > 0; d >>= 1) sum[x] += __shfl_xor(sum[x], d);
  }
  __syncthreads();
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  const float* po = a.part_o + first * 2 * D + lq * 4;
  for (int s0 = 0; s0 < nsplit; s0 += kAhead) {
    f32x4 v[kAhead][2];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s0 + i < nsplit)
#pragma unroll
        for (int x = 0; x < 2; ++x) v[i][x] = load4(po + ((s0 + i) * rows * 2 + x) * D);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s0 + i < nsplit)
#pragma unroll
        for (int x = 0; x < 2; ++x) acc[x] += wts[lr][x][s0 + i] * v[i][x];
  }
  const int token = sd.row_off + local / a.num_q_heads, head = local % a.num_q_heads;
  const float lam = a.lambda[(int64_t)token * a.lambda_stride + head];
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
  if (!live) return;
  y *= scale;
  store4(reinterpret_cast<T*>(a.out) + ((int64_t)token * a.num_q_heads + head) * D + lq * 4, y[0] * w[0], y[1] * w[1],
         y[2] * w[2], y[3] * w[3]);
}

template <typename T, int D>
void combine_as(const DiffArgs& a, hipStream_t stream) {
  const int64_t per = 256 / (D / 4);
  hipLaunchKernelGGL((diff_combine_kernel<T, D>), dim3((unsigned)((a.unit_begin[a.nseq] + per - 1) / per)), dim3(256), 0,
                     stream, a);
}

}  // namespace

hipError_t launch_diff_extend(const DiffArgs& a, int dtype, int head_dim, int grid, hipStream_t stream) {
  const dim3 g(grid), b(kThreads);
  if (dtype == 0 && head_dim == 128) hipLaunchKernelGGL((diff_extend_kernel<__bf16, 128>), g, b, 0, stream, a);
  else if (dtype == 0 && head_dim == 64) hipLaunchKernelGGL((diff_extend_kernel<__bf16, 64>), g, b, 0, stream, a);
  else if (dtype == 1 && head_dim == 128) hipLaunchKernelGGL((diff_extend_kernel<float, 128>), g, b, 0, stream, a);
  else hipLaunchKernelGGL((diff_extend_kernel<float, 64>), g, b, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_diff_combine(const DiffArgs& a, int dtype, int head_dim, hipStream_t stream) {
  if (dtype == 0 && head_dim == 128) combine_as<__bf16, 128>(a, stream);
  else if (dtype == 0 && head_dim == 64) combine_as<__bf16, 64>(a, stream);
  else if (dtype == 1 && head_dim == 128) combine_as<float, 128>(a, stream);
  else combine_as<float, 64>(a, stream);
  return hipGetLastError();
}

}  // namespace kvt
