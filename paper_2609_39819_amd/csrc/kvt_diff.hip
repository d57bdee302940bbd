// Differential attention over a paged KV cache, gfx950: a chunk of new tokens.
//
// A head's columns hold two maps of d = D/2 columns.  With K_b[j] the cached
// keys, V_b[j] the cached values and j running over the visible positions,
//   A_m = softmax_j(scale * <q_m, K_b[j]_m>),   m = 0, 1,
//   y = sum_j (A_0[j] - lambda * A_1[j]) V_b[j],
//   out = out_scale * w * y / sqrt(mean(y^2) + eps)      (w given), else out_scale * y.
// The sums of both softmaxes are known only after the last key, so one pass
// over the keys keeps an output per map: 2 D flops per (head, key) for the
// scores and 2 x 2 D for the values, in bf16 4 x 2 D (see below).
//
// Work decomposition: one workgroup per (sequence, kv-head, 128 packed query
// rows, key split), as the extend kernel's (row r = token r/G, head g*G + r%G);
// 8 waves, two per SIMD: waves 2 i and 2 i + 1 take the two maps of 32 rows each,
// on the K/V tiles that all of them share in LDS.  Row tiles of up to 64 rows
// then have a wave per SIMD (16 new tokens over 30000, 32/8 heads of 128, with one bf16
// number per probability 34.1 us; with the maps four waves apart 37.7).  A wave with
// both maps would read each V fragment once for both, but its two outputs leave no
// registers to read operands ahead (96/8 heads of 128, 1024 new tokens over 32768, one
// number per probability, 2.38 and 2.31 ms).
// S^T = K Q^T (keys on the MFMA rows, queries on the columns), so a query's scores
// sit in one lane pair (l, l+32) and leave the accumulators in the layout that the
// value product takes them in.  At the end the second map's waves hand their rows
// over through LDS and the first map's form the difference and the norm; a key
// split writes both maps' rows as they are, for the joining launch.
//
// bf16 storage: v_mfma_f32_32x32x16_bf16, tiles of 64 keys.  The value product takes
// each probability as two bf16 numbers, as the decode kernel's does: what y's two sums
// share goes, what the probabilities were rounded by would stay.  The result is then
// off by its own last rounding (2-norm, 1.66e-3 of itself).  One number each, 2^-8 of
// a probability off, leaves 2.56e-3 where the maps have nothing in common, and 1.7e-2
// where their keys differ by an eighth and lambda is 0.9 to 1; it saves a quarter to
// a third of a call.  One number for most keys and two for some is no middle way: the error is
// then that of the keys which the weight happens to lie on.
// fp32 storage: v_mfma_f32_32x32x2_f32, tiles of 32 keys, nothing rounded.
//
// What bounds it: the matrix cores with the softmax and the barriers beside them.
// A tile of 64 keys, heads of 128, takes 80 MFMAs of 32 cycles per SIMD (2560); with
// some 400 other vector instructions it lasts 4060 cycles (1.69 us) with 8 workgroups
// on the chip and 2.15 us with all CUs busy, at the clock that the board then holds.
// 2048 new tokens over 131072, 32/8 heads of 128: 8.6 ms, 11.1e12 operations, 1290
// TFLOP/s (a large bf16 matrix product 1262).  512 over 8192: 160 us.  fp32, 512 over
// 8192: 800 us, 133 TFLOP/s (a large fp32 matrix product 153).
//
// Masked positions.  Their scores are replaced by -inf, so their weight is
// exactly 0 whatever K holds; positions past the end of the sequence and unused
// page slots read the last real position instead.  But the value product
// multiplies V by that 0, and a visible position of one row is a masked one of
// another: in the tiles that reach past some row's limit a non-finite value is
// looked for first, and if there is one it is added to the rows that see it by
// hand and replaced by 0 for the product.
#include <algorithm>
#include <type_traits>

#include "kvt_diff_device.h"

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
  static constexpr int ROWB = D * (int)sizeof(T);       // bytes per key row
  static constexpr int CHUNKS = ROWB / 16;
  static constexpr int RPR = 1024 / ROWB;               // key rows per 1 KiB wave load
  static constexpr int DT = D / 32;                     // 32-wide output column tiles
  // Chunk swizzles of K and V rows.  bf16: swz (kvt_device.h).  fp32: a row is a
  // whole number of 256-byte bank cycles; a K read takes one chunk of 16 keys at
  // once, a V read half a bank cycle of one key and of the fourth after it.
  static __device__ __forceinline__ int swizzle_k(int key) {
    if constexpr (kBf16) return swz<D>(key);
    else return key & 15;
  }
  static __device__ __forceinline__ int swizzle_v(int key) {
    if constexpr (kBf16) return swz<D>(key);
    else return (key & 4) << 1;
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

// One K or V tile.
template <typename T, int D>
struct HalfTile {
  T e[Shape<T, D>::KT * D];
};

// A wave's query rows, its map's half of the columns, as the B operand of the
// score product.  bf16: fragment k holds columns 16 k + 8 hh .. + 7.  fp32:
// element i of fragment k is column 8 k + 4 hh + i.
template <typename T, int D>
struct Queries;
template <int D>
struct Queries<__bf16, D> {
  bf16x8 f[D / 32];
  __device__ __forceinline__ void load(const __bf16* p, int hh) {
#pragma unroll
    for (int k = 0; k < D / 32; ++k) f[k] = __builtin_bit_cast(bf16x8, load8(p + k * 16 + hh * 8));
  }
};
template <int D>
struct Queries<float, D> {
  f32x4 f[D / 16];
  __device__ __forceinline__ void load(const float* p, int hh) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) f[k] = load4(p + k * 8 + hh * 4);
  }
};

// bf16 heads of 64 hold to 128 registers and share a CU between two workgroups
// (4096 new tokens over 16384, 32/8 heads: 1650 us one to a CU, 1480 two).
template <typename T, int D>
__global__ __launch_bounds__(kThreads, (D == 64 && sizeof(T) == 2) ? 4 : 2) void diff_extend_kernel(const DiffArgs a) {
  using S = Shape<T, D>;
  constexpr int KT = S::KT, DT = S::DT, RPR = S::RPR;
  constexpr int PAGES = KT / kBlock;                              // pages per tile
  constexpr int NREG = KT * S::ROWB / 1024 / kDiffWaves;          // 1 KiB loads per wave per tensor
  constexpr int QK = S::kBf16 ? D / 32 : D / 16;                  // query fragments
  constexpr int KG = S::kBf16 ? 2 : 16;                           // key groups of the value product over 32 keys
  constexpr float kRescaleSlack = 8.0f;                           // log2 headroom before O is rescaled
  constexpr float kSumLimit = 65536.0f;                           // a lane's sum of probabilities over 32 keys
  struct Probs {   // B operands of the value product over 32 keys; bf16: a probability is w + rest
    typename std::conditional<S::kBf16, u32x4, float>::type w[KG];
    u32x4 rest[S::kBf16 ? KG : 1];
  };
  typedef typename std::conditional<S::kBf16, bf16x8, float>::type VFrag;
  // rings of four K and four V tiles; distinct objects, so that the compiler can
  // tell the page gather into one from the operand reads of another
  __shared__ __attribute__((aligned(1024))) HalfTile<T, D> k0, k1, k2, k3, v0, v1, v2, v3;
  __shared__ float row_sum[kDiffTileRows];   // of the second map, for the epilogue
  __shared__ int odd_seen;                   // a non-finite value was found in a tile with masked positions

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int map = wave & 1, rg = wave >> 1;   // this wave's map and 32-row block
  const int hh = lane >> 5;     // lane half
  const int l32 = lane & 31;
  if (tid == 0) odd_seen = 0;

  // ---- which (sequence, kv-head, row tile, key split) this workgroup owns
  const int hkv = a.num_kv_heads;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const int si = find_seq(a.unit_begin, a.nseq, unit);
  const SeqDesc sd = a.seq[si];
  const int nsplit = a.nsplit[si], nlast = a.nlast[si];
  const int local = unit - a.unit_begin[si];
  const int G = a.group;
  const int rows_seq = sd.suffix * G;
  const int ntile = (rows_seq + kDiffTileRows - 1) / kDiffTileRows;
  // longest (last) row tile first
  const bool last = local < nlast;
  const int rt = last ? ntile - 1 : ntile - 2 - (local - nlast) / nsplit;
  const int split = last ? local : (local - nlast) % nsplit;
  const int r0 = rt * kDiffTileRows;
  const int P = sd.prefix;
  const int L = P + sd.suffix;                 // positions that can be read
  const int nblk = (L + kBlock - 1) / kBlock;

  // keys up to the tile's last query's own position, evenly over the splits
  const int t_last = min(sd.suffix - 1, (r0 + kDiffTileRows - 1) / G);
  const int ntiles_kv = (P + t_last + KT) / KT;
  const int per_split = last ? (ntiles_kv + nlast - 1) / nlast : (ntiles_kv + nsplit - 1) / nsplit;
  const int j0 = split * per_split;
  const int j1 = min(ntiles_kv, j0 + per_split);
  const int n = j1 - j0;                       // tiles (none: a split past the keys)
  const int masked = max(0, (P + r0 / G + 1) / KT - j0);   // first one with positions that some row does not see

  // ---- this lane's query row
  const bool idle = r0 + rg * 32 >= rows_seq;  // a wave past the last row only takes part in the gather
  const int r = min(r0 + rg * 32 + l32, rows_seq - 1);
  const bool row_valid = r0 + rg * 32 + l32 < rows_seq;
  const int t_row = r / G;
  const int h_row = g * G + (r - t_row * G);
  const int lim = P + t_row;                   // last visible position
  const int64_t qrow = (int64_t)(sd.row_off + t_row) * a.num_q_heads + h_row;
  Queries<T, D> q;
  q.load(reinterpret_cast<const T*>(a.q) + qrow * D + map * (D / 2), hh);

  const char* kpool = reinterpret_cast<const char*>(a.k_pool);
  const char* vpool = reinterpret_cast<const char*>(a.v_pool);
  // read-only here: a constant-address-space view lets wave-uniform page
  // lookups become scalar loads
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;

  // ---- gather geometry: a wave's NREG loads of a tile lie in one page, so it
  // looks up one page id per tile.  Load i covers key rows RPR*(NREG*w + i) ..
  // +RPR-1; lane l lands at LDS byte 16*l of that 1 KiB run, i.e. row l/CHUNKS,
  // physical chunk l%CHUNKS, so it fetches logical chunk (l%CHUNKS) ^ swizzle(row).
  const int page_in_tile = wave * PAGES / kDiffWaves;
  uint32_t k_off[NREG], v_off[NREG];           // this lane's byte offset within its page run
#pragma unroll
  for (int i = 0; i < NREG; ++i) {
    const int key = RPR * (wave * NREG + i) + lane / S::CHUNKS;
    const int row = (key & (kBlock - 1)) * S::ROWB, chunk = lane % S::CHUNKS;
    k_off[i] = (uint32_t)(row + ((chunk ^ S::swizzle_k(key)) << 4));
    v_off[i] = (uint32_t)(row + ((chunk ^ S::swizzle_v(key)) << 4));
  }
  // page id as the block table has it, clamped into the pool where it is used
  auto page_id = [&](int jn) __attribute__((always_inline)) {
    return (uint32_t)bt[__builtin_amdgcn_readfirstlane(min(jn * PAGES + page_in_tile, nblk - 1))];
  };
  // positions past the end of the sequence take the last real position's offset
  const uint32_t tail = (uint32_t)((L - 1) & (kBlock - 1)) * S::ROWB;
  auto gather = [&](const char* pool, const uint32_t (&lane_off)[NREG], int jn, uint32_t id, HalfTile<T, D>& dst)
      __attribute__((always_inline)) {
    const uint32_t last = jn * PAGES + page_in_tile >= nblk - 1 ? tail : (kBlock - 1) * S::ROWB;
    const char* base = pool + (((int64_t)min(id, nb_max) * hkv + g) << 4) * S::ROWB;
#pragma unroll
    for (int i = 0; i < NREG; ++i)
      __builtin_amdgcn_global_load_lds((const void*)(base + min(lane_off[i], last | (lane_off[i] & (S::ROWB - 1)))),
                                       (lds_void*)((lds_char*)dst.e + (wave * NREG + i) * 1024), 16, 0, 0);
  };

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = (f32x16){};
  float m_ref = -INFINITY, m_neg = NAN, l_run = 0.f;   // reference max of scale*log2e*score; this lane's share of sum 2^(s*c - m_ref)
  const float c = a.scale_log2;

  // ---- S^T = K Q^T: product k of a 32-key block takes 16 of the map's columns (fp32: 8)
  int k_at[QK];   // this lane's byte offset in a K tile
#pragma unroll
  for (int k = 0; k < QK; ++k) k_at[k] = l32 * S::ROWB + (((2 * (map * QK + k) + hh) ^ S::swizzle_k(l32)) << 4);
  auto read_k = [&](const HalfTile<T, D>& tl, int k, int half) __attribute__((always_inline)) {
    return *(const lds_u32x4*)((const lds_char*)tl.e + half * 32 * S::ROWB + k_at[k]);
  };
  auto score_product = [&](u32x4 kf, int k, f32x16 acc) __attribute__((always_inline)) {
    if constexpr (S::kBf16) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), q.f[k], acc, 0, 0, 0);
    } else {
      const f32x4 k4 = __builtin_bit_cast(f32x4, kf);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(k4[i], q.f[k][i], acc, 0, 0, 0);
      return acc;
    }
  };
  // ---- causal mask of 32 keys from `first` on.  Element e is key first + 8 (e/4) + 4 hh + e%4.
  auto mask = [&](int first, f32x16& s) __attribute__((always_inline)) {
    const int thr = lim - first - 4 * hh;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (8 * (e >> 2) + (e & 3) > thr) s[e] = -INFINITY;
  };
  // ---- moves the reference to the row maxima of these scores where they pass it
  // by more than the slack; returns the factor for what was summed before.  m_neg,
  // which the probabilities are formed with, is NaN until the row has a reference:
  // their sum then tells check
  auto settle = [&](const f32x16& s) __attribute__((always_inline)) {
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
    const float mxc = pair_max(mx) * c;
    const float m_new = (mxc > m_ref + kRescaleSlack) ? mxc : m_ref;
    // 1 when unchanged, 0 when leaving -inf; kept at 1 while the row has seen no visible key
    const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m_ref - m_new);
    m_ref = m_new;
    m_neg = (m_ref == -INFINITY) ? NAN : -m_ref;
    return alpha;
  };
  // ---- probabilities of 32 keys as B operands of the value product; returns their
  // sum
  auto probs = [&](const f32x16& s, Probs& p, float neg) __attribute__((always_inline)) {
    float rs = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, neg));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], c, neg));
      if constexpr (S::kBf16) {
        unsigned w, rest;
        two_numbers(p0, p1, w, rest);
        p.w[i / 8][i % 8 / 2] = w;
        p.rest[i / 8][i % 8 / 2] = rest;
      } else {
        p.w[i] = p0;
        p.w[i + 1] = p1;
      }
      rs += p0 + p1;
    }
    return rs;
  };
  // ---- O^T += V^T P^T: product kg takes 16 keys (fp32: keys 8 (kg/4) + kg%4 and the
  // fourth after it, one per lane half) of 32 columns
  const int g16 = (lane >> 4) & 1, rsel = (lane & 15) >> 2;
  // bf16: this lane's byte offsets in a V tile; with the bias in them what is left to
  // add fits the 16 bits of a read's immediate offset where the K slots take 64 KiB
  constexpr int kBias = 4 * sizeof(HalfTile<T, D>) >= 65536 ? 65536 : 0;
  int v_at[2][DT];
#pragma unroll
  for (int r2 = 0; r2 < 2; ++r2)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int key = 8 * r2 + 4 * hh + rsel;            // key within a 16-key group
      const int dcol = dt * 32 + g16 * 16 + 4 * (lane & 3);
      v_at[r2][dt] = (key * D + (((dcol >> 3) ^ S::swizzle_v(key)) << 3) + (dcol & 7)) * (int)sizeof(T) + kBias;
    }
  auto read_v = [&](const HalfTile<T, D>& tl, int half, int kg, int dt) __attribute__((always_inline)) {
    if constexpr (S::kBf16) {
      bf16x4 v[2];
#pragma unroll
      for (int r2 = 0; r2 < 2; ++r2)
        v[r2] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (lds_bf16x4*)((const lds_char*)tl.e + (v_at[r2][dt] + ((half * 32 + kg * 16) * S::ROWB - kBias))));
      return (VFrag)__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int key = 8 * (kg >> 2) + 4 * hh + (kg & 3), col = dt * 32 + l32;
      return (VFrag)tl.e[key * D + (((col >> 2) ^ S::swizzle_v(key)) << 2) + (col & 3)];
    }
  };
  auto value_product = [&](VFrag vf, const Probs& p, int kg, f32x16 acc) __attribute__((always_inline)) {
    if constexpr (S::kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p.w[kg]), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x2f32(vf, p.w[kg], acc, 0, 0, 0);
  };
  auto rest_product = [&](VFrag vf, const Probs& p, int kg, f32x16 acc) __attribute__((always_inline)) {
    if constexpr (S::kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, p.rest[kg]), acc, 0, 0, 0);
    else return acc;
  };

  // ---- non-finite values in a V tile with masked positions (see the top) become
  // 0 there; any_odd (workgroup-uniform) remembers it
  bool any_odd = false;
  constexpr int VPIECES = KT * S::ROWB / 16 / kThreads;   // 16-byte pieces of a tile per thread
  auto drop_odd = [&](HalfTile<T, D>& tl) __attribute__((always_inline)) {
    u32x4* p = reinterpret_cast<u32x4*>(tl.e) + tid;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < VPIECES; ++i) {
      const u32x4 w = p[kThreads * i];
#pragma unroll
      for (int x = 0; x < 4; ++x) odd = odd || non_finite<T>(w[x]);
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0 && lane == 0) odd_seen = 1;
    __syncthreads();
    if (odd_seen == 0) return;
    any_odd = true;
#pragma unroll
    for (int i = 0; i < VPIECES; ++i) {
      u32x4 w = p[kThreads * i];
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = finite_part<T>(w[x]);
      p[kThreads * i] = w;
    }
    __syncthreads();
  };

  auto score_block = [&](const HalfTile<T, D>& tl, int half, f32x16& s) __attribute__((always_inline)) {
    s = (f32x16){};
#pragma unroll
    for (int k = 0; k < QK; ++k) s = score_product(read_k(tl, k, half), k, s);
  };
  auto value_block = [&](const HalfTile<T, D>& tl, int half, const Probs& p) __attribute__((always_inline)) {
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) {
      VFrag vf[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        vf[dt] = read_v(tl, half, kg, dt);
        o[dt] = value_product(vf[dt], p, kg, o[dt]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = rest_product(vf[dt], p, kg, o[dt]);
    }
  };
  // whether the probabilities p of the scores s hold; rs: their sum.  Where the
  // reference is not set yet, or some score passed it by far, or is a NaN, they
  // are done again from the row maxima (a row that still sees nothing has weights 0).
  auto check = [&](const f32x16& s, Probs& p, float rs) __attribute__((always_inline)) {
    if (__builtin_amdgcn_ballot_w64(!(rs < kSumLimit)) != 0) {
      const float alpha = settle(s);
      rs = probs(s, p, m_ref == -INFINITY ? 0.f : -m_ref);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
    }
    l_run += rs;
  };
  // bf16, 32 keys: probabilities of `cur` while the matrix cores form the scores of
  // the next 32 keys and the value product of the 32 before, three streams that
  // do not depend on each other.  Heads of 128 read the K fragments of those scores
  // in the turn before (kf; kt, khalf is the block of the turn after), so that a
  // turn's first products have nothing to wait for (4 % of a tile).  With heads of
  // 64, whose scores take two products, that costs 5 %: kt, khalf is this turn's block.
  constexpr bool kReadAhead = D == 128;
  u32x4 kf[QK];
  auto turn = [&](const HalfTile<T, D>& kt, int khalf, const f32x16& cur, f32x16& next, const HalfTile<T, D>& vt, int vhalf,
                  const Probs& prev, Probs& out) __attribute__((always_inline)) {
    if constexpr (kReadAhead) {
      next = (f32x16){};
#pragma unroll
      for (int k = 0; k < QK; ++k) next = score_product(kf[k], k, next);
    } else {
      score_block(kt, khalf, next);
    }
    value_block(vt, vhalf, prev);
    if constexpr (kReadAhead) {
#pragma unroll
      for (int k = 0; k < QK; ++k) kf[k] = read_k(kt, k, khalf);
    }
    const float rs = probs(cur, out, m_neg);
    // after each product two operand reads and a share of the softmax
#pragma unroll
    for (int i = 0; i < QK + 2 * KG * DT; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, kReadAhead ? 2 : 8, 0);
    }
    check(cur, out, rs);
  };

  // ---- main loop: step t takes tile t.  K of tile t+3 and V of tile t+2 start to
  // stream in, each into the slot that the step before was done with (past the
  // last tile the gather reads clamped, in-bounds pages into slots no one reads).
  // They are waited for before the barrier at the end (each wave counts its own loads
  // only): a step is longer than a load takes, and a barrier that left them in flight
  // measured the same.
  // bf16: the scores of a tile's first half come from the step before, and the
  // value product of its second half is left to the step after.
  uint32_t id2 = page_id(j0 + 2), id3 = page_id(j0 + 3);   // pages of tiles t+2, t+3
  f32x16 s0, s1;
  Probs p0, p1;
  if (n > 0) {
    const uint32_t id0 = page_id(j0), id1 = page_id(j0 + 1);
    gather(kpool, k_off, j0, id0, k0);
    gather(vpool, v_off, j0, id0, v0);
    gather(kpool, k_off, j0 + 1, id1, k1);
    gather(kpool, k_off, j0 + 2, id2, k2);
    gather(vpool, v_off, j0 + 1, id1, v1);
  }
  if constexpr (S::kBf16) {
    // nothing before the first tile: probabilities and values of 0
#pragma unroll
    for (int i = 0; i < KG; ++i) p1.w[i] = p1.rest[i] = (u32x4){0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < VPIECES; ++i) reinterpret_cast<u32x4*>(v3.e)[tid + kThreads * i] = (u32x4){0u, 0u, 0u, 0u};
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  __syncthreads();
  if (S::kBf16 && n > 0 && !idle) {
    score_block(k0, 0, s0);
    if (masked == 0) mask(j0 * KT, s0);
    settle(s0);
    if constexpr (kReadAhead) {
#pragma unroll
      for (int k = 0; k < QK; ++k) kf[k] = read_k(k0, k, 1);
    }
  }
  auto step = [&](int t, const HalfTile<T, D>& k_cur, const HalfTile<T, D>& k_next, const HalfTile<T, D>& v_prev,
                  HalfTile<T, D>& v_cur, HalfTile<T, D>& k_fill, HalfTile<T, D>& v_fill) __attribute__((always_inline)) {
    gather(kpool, k_off, j0 + t + 3, id3, k_fill);
    gather(vpool, v_off, j0 + t + 2, id2, v_fill);
    id2 = id3, id3 = page_id(j0 + t + 4);
    if (t >= masked) drop_odd(v_cur);
    // opaque, so that the slots' bases go into the reads' immediate offsets and not
    // into a register for each slot and offset (46 registers)
    if constexpr (S::kBf16) {
#pragma unroll
      for (int k = 0; k < QK; ++k) asm("" : "+v"(k_at[k]));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) asm("" : "+v"(v_at[0][dt]), "+v"(v_at[1][dt]));
    }
    if (!idle) {
      // asm: a branch where there is something to mask, not selects on every tile
      if constexpr (S::kBf16) {
        if (t >= masked) {
          asm volatile("");
          mask((j0 + t) * KT, s0);
        }
        turn(kReadAhead ? k_next : k_cur, kReadAhead ? 0 : 1, s0, s1, v_prev, 1, p1, p0);
        if (t >= masked) {
          asm volatile("");
          mask((j0 + t) * KT + 32, s1);
        }
        turn(k_next, kReadAhead ? 1 : 0, s1, s0, v_cur, 0, p0, p1);
      } else {
        score_block(k_cur, 0, s0);
        if (t >= masked) {
          asm volatile("");
          mask((j0 + t) * KT, s0);
        }
        check(s0, p0, probs(s0, p0, m_neg));
        value_block(v_cur, 0, p0);
      }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __syncthreads();
  };
  for (int t = 0; t < n; t += 4) {
    step(t, k0, k1, v3, v0, k3, v2);
    if (t + 1 >= n) break;
    step(t + 1, k1, k2, v0, v1, k0, v3);
    if (t + 2 >= n) break;
    step(t + 2, k2, k3, v1, v2, k1, v0);
    if (t + 3 >= n) break;
    step(t + 3, k3, k0, v2, v3, k2, v1);
  }
  if (S::kBf16 && n > 0 && !idle) {
    const HalfTile<T, D>& v_last = (n & 3) == 1 ? v0 : (n & 3) == 2 ? v1 : (n & 3) == 3 ? v2 : v3;
    value_block(v_last, 1, p1);
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  // what drop_odd left out: the rows that see such a value get it by hand
  if (any_odd && !idle) {
    for (int pos = (j0 + masked) * KT; pos < min(j1 * KT, L); ++pos) {
      const uint32_t id = min((uint32_t)bt[pos / kBlock], nb_max);
      const T* vr = reinterpret_cast<const T*>(vpool) + ((((int64_t)id * hkv + g) << 4) + (pos & (kBlock - 1))) * D;
      bool odd = false;
      for (int w = lane; w < S::ROWB / 4; w += 64) odd = odd || non_finite<T>(reinterpret_cast<const unsigned*>(vr)[w]);
      if (__builtin_amdgcn_ballot_w64(odd) == 0) continue;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float v = (float)vr[dt * 32 + 8 * (e >> 2) + 4 * hh + (e & 3)];
          if (pos <= lim && !__builtin_isfinite(v)) o[dt][e] += v;
        }
    }
  }

  // ---- epilogue
  const float l_tot = pair_sum(l_run) * (S::kBf16 ? kOver : 1.0f);
  if (nsplit > 1) {
    if (!row_valid) return;
    const int64_t rows = (int64_t)sd.suffix * a.num_q_heads;
    const int64_t prow = a.part_row[si] + split * rows + (int64_t)t_row * a.num_q_heads + h_row;
    float* op = a.part_o + (prow * 2 + map) * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = dt * 32 + 8 * i + 4 * hh;
        store4(op + d, o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]);
      }
    if (hh == 0) *reinterpret_cast<f32x2*>(a.part_ml + prow * 4 + 2 * map) = (f32x2){m_ref, l_tot};
    return;
  }
  // the second map's waves hand their rows over through the rings, a block per
  // ring slot, the 16-byte pieces of a row XOR-swizzled
  static_assert(sizeof(HalfTile<T, D>) >= 32 * D * sizeof(float), "hand-over buffer");
  constexpr int Q4 = D / 4;
  f32x4* hand = reinterpret_cast<f32x4*>(rg == 0 ? k0.e : rg == 1 ? k1.e : rg == 2 ? v0.e : v1.e) + l32 * Q4;
  __syncthreads();   // the last value products have read the rings
  if (map == 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        hand[(dt * 8 + 2 * i + hh) ^ (l32 & (Q4 - 1))] =
            (f32x4){o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
    if (hh == 0) row_sum[rg * 32 + l32] = l_tot;
  }
  __syncthreads();
  if (map == 1) return;
  const float lam = a.lambda[(int64_t)(sd.row_off + t_row) * a.lambda_stride + h_row];
  const float inv0 = 1.0f / l_tot, inv1 = 1.0f / row_sum[rg * 32 + l32];
  float sq = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 o1 = hand[(dt * 8 + 2 * i + hh) ^ (l32 & (Q4 - 1))];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float y = map_difference(o[dt][4 * i + x], inv0, o1[x], inv1, lam);
        o[dt][4 * i + x] = y;
        sq += y * y;
      }
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
      store4(op + d, o[dt][4 * i] * scale * w[0], o[dt][4 * i + 1] * scale * w[1], o[dt][4 * i + 2] * scale * w[2],
             o[dt][4 * i + 3] * scale * w[3]);
    }
}

// Joins the key splits of each row (fixed order): with m* = max_s m_s and
// w_s = 2^(m_s - m*), map m is sum_s w_s O_s / sum_s w_s l_s; then the maps'
// difference and its norm as in the kernel's own epilogue.  A group of D/4 lanes
// holds a row, four columns a lane (GROUPS > 1: that many groups share the row's
// splits, and a workgroup holds one row); the weights of the splits are formed once
// per row, one split per lane, and shared through LDS.  Every split is multiplied by
// its weight, be it 0, so an infinity or a NaN among the values gives the unsplit
// call's.  args: the sequences with more than one split; unit_begin counts their
// rows.
constexpr int kAhead = 4;   // splits whose pieces are in flight at once, the first from before the weights are known

template <typename T, int D, int GROUPS>
__global__ __launch_bounds__(256) void diff_combine_kernel(const DiffArgs a) {
  constexpr int Q4 = D / 4, ROWS = 256 / Q4 / GROUPS;   // lanes of a group, rows per workgroup
  constexpr int PER = (kMaxPartials + Q4 - 1) / Q4;
  __shared__ float wts[ROWS][2][kMaxPartials];
  __shared__ f32x4 part[GROUPS > 1 ? GROUPS : 1][2][Q4];
  const int lr = threadIdx.x / (Q4 * GROUPS), grp = threadIdx.x / Q4 % GROUPS, lq = threadIdx.x % Q4;
  const int total = a.unit_begin[a.nseq];
  const int idx = blockIdx.x * ROWS + lr;
  const bool live = idx < total;
  const int row = live ? idx : total - 1;
  const int si = find_seq(a.unit_begin, a.nseq, row);
  const SeqDesc sd = a.seq[si];
  const int local = row - a.unit_begin[si];        // token * Hq + head within the sequence
  const int packed = local / a.num_q_heads * a.group + local % a.num_q_heads % a.group;
  const int nsplit = packed / kDiffTileRows == (sd.suffix * a.group - 1) / kDiffTileRows ? a.nlast[si] : a.nsplit[si];
  const int64_t rows = (int64_t)sd.suffix * a.num_q_heads;
  const int64_t first = a.part_row[si] + (int64_t)local;

  const float* po = a.part_o + first * 2 * D + lq * 4;
  f32x4 v[kAhead][2];
  auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s0 + i * GROUPS < nsplit)
#pragma unroll
        for (int x = 0; x < 2; ++x) v[i][x] = load4(po + ((s0 + i * GROUPS) * rows * 2 + x) * D);
  };
  load(grp);
  const int token = sd.row_off + local / a.num_q_heads, head = local % a.num_q_heads;
  const float lam = a.lambda[(int64_t)token * a.lambda_stride + head];
  f32x4 w = {1.f, 1.f, 1.f, 1.f};
  if (a.norm_weight != nullptr) w = load4(a.norm_weight + lq * 4);
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
      const float ws = (m[x][k] == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m[x][k] - top[x]);
      sum[x] += ws * l[x][k];
      if (s < nsplit && grp == 0) wts[lr][x][s] = ws;
    }
#pragma unroll
    for (int d = Q4 / 2; d > 0; d >>= 1) sum[x] += __shfl_xor(sum[x], d);
  }
  __syncthreads();
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  for (int s0 = grp; s0 < nsplit; s0 += kAhead * GROUPS) {
    if (s0 >= GROUPS) load(s0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s0 + i * GROUPS < nsplit)
#pragma unroll
        for (int x = 0; x < 2; ++x) acc[x] += wts[lr][x][s0 + i * GROUPS] * v[i][x];
  }
  if constexpr (GROUPS > 1) {   // one row: the groups' shares, in order
#pragma unroll
    for (int x = 0; x < 2; ++x) part[grp][x][lq] = acc[x];
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) acc[x] += part[i][x][lq];
  }
  const float inv0 = 1.0f / sum[0], inv1 = 1.0f / sum[1];
  f32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = map_difference(acc[0][i], inv0, acc[1][i], inv1, lam);
  float scale = a.out_scale;
  if (a.norm_weight != nullptr) {
    float sq = y[0] * y[0] + y[1] * y[1] + y[2] * y[2] + y[3] * y[3];
#pragma unroll
    for (int d = Q4 / 2; d > 0; d >>= 1) sq += __shfl_xor(sq, d);
    scale *= 1.0f / __builtin_sqrtf(sq * (1.0f / D) + a.eps);
  }
  if (!live) return;
  y *= scale;
  store4(reinterpret_cast<T*>(a.out) + ((int64_t)token * a.num_q_heads + head) * D + lq * 4, y[0] * w[0], y[1] * w[1],
         y[2] * w[2], y[3] * w[3]);
}

template <typename T, int D>
void combine_as(const DiffArgs& a, hipStream_t stream) {
  constexpr int kGroups = 256 / (D / 4);
  const int rows = a.unit_begin[a.nseq], splits = *std::max_element(a.nsplit, a.nsplit + a.nseq);
  // a whole workgroup per row pays where a chain of loads is what a row waits for:
  // decode, 96 rows of 22 splits 90.2 us a call with a group per row, 87.5 so; 32 of
  // 22 17.5 and 15.1; extend, 512 rows of 32 34.2 and 33.0; but 1024 rows of 8 29.6 and
  // 30.3, 2144 of 11 81.1 and 84.7
  const bool wide = splits > 2 * kAhead && rows <= 1024;
  if (wide) hipLaunchKernelGGL((diff_combine_kernel<T, D, kGroups>), dim3(rows), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((diff_combine_kernel<T, D, 1>), dim3((rows + kGroups - 1) / kGroups), dim3(256), 0, stream, a);
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
