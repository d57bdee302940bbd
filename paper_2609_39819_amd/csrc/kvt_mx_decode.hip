// Attention of few query rows over 4-bit pages, gfx950: a decoding step, or chunks
// of up to 64 rows (new tokens x query heads) of a kv-head.
//
// The formula is kvt_decode.hip's, with a last visible position for each row; the cost is streaming each sequence's 4-bit
// K/V once from HBM (2 * 17/32 D bytes a key and kv-head).  Work decomposition:
//   * the batch's 32-key tiles lie one after the other, and one workgroup per (equal
//     share of them, kv-head, up to 32 of the kv-head's rows) goes through
//     the parts of sequences in its share; of each, wave w of 4 takes the tiles w,
//     w+4, .. and keeps two of them in flight in registers, across the sequences'
//     borders; no barrier in the loop;
//   * v_mfma_f32_16x16x32_bf16 with 16 rows (NB = 1) or 32 (NB = 2): S^T = K Q^T.
//     A lane's K operand is 8 columns of one key, in any order of the columns
//     that Q's shares, so each lane takes D/4 neighbouring columns of its key:
//     16 bytes of codes under one scale (D = 128), converted straight into the
//     operand.  K never goes through LDS;
//   * V does, as bf16 [key][D], because its operand runs along the keys: the
//     lane that loaded 32 columns of a key writes them, and transposed reads
//     bring them back; the rows are swizzled so that neither has a conflict;
//   * fp32 queries are three bf16 terms, and so are the probabilities: every
//     product then keeps fp32's 24 bits (the 4-bit values are exact in bf16);
//   * at the end the four waves' (m, l, O) merge through LDS into the output or
//     a partial of the key split.
//
// Measured, bf16 queries: one context of 131072 keys, 96/8 heads of 128, 143 MB,
// 32.7 us with the join (4.4 TB/s; the first tiles and the join's launch are
// about 8 us of it), 64 contexts of 1024..16384 83 us (5.1 TB/s; a plain read of
// 2 GiB 6.1; this kernel's loads alone 78.6), heads of 64 57 us (3.7 TB/s, its loads
// alone 52: pages of half the bytes in as many places).  Messages of 2, 8 and 16
// tokens over 131000 keys, 32/8 heads: 33.0, 50.4 and 67.4 us; by the extend kernel
// 93.7, 94.6 and 97.8.  With fp32 queries, 32/8 heads: one context of 131072 36.7 us, 64
// of 1024..16384 98.8.
#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

constexpr int kWaves = kDecWaves;
constexpr int kTK = kDecKeysPerTile;   // keys per tile = 2 pages

// A wave's V tile, [key][D] bf16, and its O rows for the merge, [row][D] fp32:
// with 16 rows in a place of their own, so that a wave starts on the next sequence
// while others still merge.
template <int D, int NB>
struct alignas(1024) MxDecSlot {
  static constexpr bool kApart = NB == 1;
  char v[kTK * D * 2 > (kApart ? 0 : NB * 16 * D * 4) ? kTK * D * 2 : NB * 16 * D * 4];
  char own[kApart ? NB * 16 * D * 4 : 16];
  __device__ f32x4* rows() { return reinterpret_cast<f32x4*>(kApart ? own : v); }
};

// XOR swizzle of the 16-byte chunks of a V row in LDS.  A write takes 16 keys at
// one chunk, a transposed read 8 keys at two neighbouring chunks (the first an
// even one): both get 16 distinct bank groups of the 256 bytes of a cycle.
template <int D>
__device__ __forceinline__ int swz_mx(int key) {
  if constexpr (D == 128) return ((key & 7) << 1) | ((key >> 3) & 1);
  else return (((key >> 1) & 3) << 1) | ((key >> 3) & 1);
}

// STEP: one new token per sequence, which sees all of it.
template <typename T, int D, int NB, bool STEP>
__global__ __launch_bounds__(kWaves * 64, sizeof(T) == 4 && D == 128 && NB == 2 ? 1 : 2) void mx_decode_kernel(const MxDecodeArgs a) {
  constexpr int NT = kTerms<T>;
  constexpr int KS = D / 32;                     // score steps = words of a lane's codes
  constexpr int CT = D / 16;                     // 16-column tiles of the output
  constexpr int64_t kPage = mx_page_bytes(D);
  constexpr float kRescaleSlack = 8.0f;
  __shared__ MxDecSlot<D, NB> ring[kWaves];
  __shared__ float ml[kWaves][NB * 16][2];       // per wave and row: m (log2 units), l

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15;
  const int qd = lane >> 4;

  // ---- which kv-head, rows and tiles this workgroup owns (row r of a sequence is
  // token r / G, head g * G + r % G)
  const int hkv = a.num_kv_heads;
  const int G = a.group;
  const int heads = hkv * a.chunks;
  const Place8 at8 = place_of(blockIdx.x, gridDim.x, heads);
  const int unit = at8.unit;
  const int g = at8.head % hkv;
  const int r0 = at8.head / hkv * NB * 16;       // this workgroup's rows of a sequence start here
  const int share = a.share;
  const char* kpool = reinterpret_cast<const char*>(a.k_pool);
  const char* vpool = reinterpret_cast<const char*>(a.v_pool);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
  __bf16* vs = reinterpret_cast<__bf16*>(ring[wave].v);
  const lds_bf16* vl = (const lds_bf16*)vs;
  const int vkey = 4 * qd + (l16 >> 2);          // key of this lane's transposed reads
  const int vrow = vkey * D + (l16 & 1) * 4, vsub = (l16 >> 1) & 1, vswz = swz_mx<D>(vkey);
  const float c = a.scale_log2;

  int si = share == 0 ? unit : find_seq(a.tile_begin, a.nseq, unit * share);
  int from = share == 0 ? a.tile_begin[si] : unit * share;
  const int to = share == 0 ? a.tile_begin[si + 1] : min(from + share, a.tile_begin[a.nseq]);

  // ---- where the loads are: tile `j` of the sequence, this wave's next one in
  // the slot.  They run ahead of the products across the sequences' borders, so
  // that a short sequence does not wait for its first tiles.
  typedef const __attribute__((address_space(4))) int32_t* Ids;
  struct Place {
    int si, j, j1, L, nblk;
    Ids bt;
  } at;
  auto enter = [&](int x, int first_tile) __attribute__((always_inline)) {
    const SeqDesc sd = a.seq[x];
    at.si = x;
    at.L = sd.prefix + sd.suffix;
    at.nblk = (at.L + kBlock - 1) / kBlock;
    at.j = first_tile - a.tile_begin[x] + wave;
    at.j1 = STEP || sd.suffix * G > r0 ? min(to, a.tile_begin[x + 1]) - a.tile_begin[x] : 0;   // 0: no rows, no tiles
    at.bt = (Ids)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  };
  // the next tile with work for this wave; past the last one its place stays (on
  // a tile of the slot's last sequence)
  auto settle = [&]() __attribute__((always_inline)) {
    while (at.j >= at.j1 && a.tile_begin[at.si + 1] < to) enter(at.si + 1, a.tile_begin[at.si + 1]);
    at.j = STEP ? min(at.j, at.j1 - 1) : max(0, min(at.j, at.j1 - 1));
  };
  enter(si, from);
  settle();
  uint32_t ids[2];                               // its pages
  auto page_ids = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = __builtin_amdgcn_readfirstlane(min(at.j * 2 + p, at.nblk - 1));
      ids[p] = (uint32_t)at.bt[page];
    }
  };
  // one tile in flight: per page, the lane's codes and scales of key l16
  struct Stage {
    unsigned k[2][KS], v[2][KS];
    unsigned char sk[2], sv[2];
  };
  // the tile at `at`, which moves on; positions past the sequence's end read the
  // last real position (weight 0)
  auto load_tile = [&](Stage& st) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = min(at.j * 2 + p, at.nblk - 1);
      const int slot = min(l16, at.L - 1 - page * kBlock);
      const int64_t record = ((int64_t)min(ids[p], nb_max) * hkv + g) * kPage;
      const int code = slot * (D / 2) + qd * (D / 8);
      const int scale = mx_code_bytes(D) + slot * (D / 32) + (D == 128 ? qd : qd >> 1);
      const char* ks = kpool + record;
      const char* vs = vpool + record;
      if constexpr (KS == 4) {
        const u32x4 k4 = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(ks + code));
        const u32x4 v4 = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vs + code));
#pragma unroll
        for (int i = 0; i < 4; ++i) st.k[p][i] = k4[i], st.v[p][i] = v4[i];
      } else {
        const u32x2 k2 = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(ks + code));
        const u32x2 v2 = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(vs + code));
#pragma unroll
        for (int i = 0; i < 2; ++i) st.k[p][i] = k2[i], st.v[p][i] = v2[i];
      }
      st.sk[p] = (unsigned char)ks[scale];
      st.sv[p] = (unsigned char)vs[scale];
    }
    at.j += kWaves;
    settle();
    page_ids();
  };

  // ---- this lane's query rows (rows past the last repeat it and are dropped):
  // columns qd * D/4 .., and the last position each sees
  bf16x8 qreg[NB][KS][NT];
  int lim[STEP ? 1 : NB];
  auto load_rows = [&](int x) __attribute__((always_inline)) {
    const SeqDesc sd = a.seq[x];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const unsigned r = min(r0 + b * 16 + l16, (STEP ? G : sd.suffix * G) - 1), t = STEP ? 0u : r / (unsigned)G;
      const int64_t row = (int64_t)(sd.row_off + (int)t) * a.num_q_heads + g * G + (int)(r - t * G);
      const T* qp = reinterpret_cast<const T*>(a.q) + row * D + qd * (D / 4);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) load_terms(qp + kk * 8, qreg[b][kk]);
      if constexpr (!STEP) lim[b] = sd.prefix + (int)t;
    }
  };

  f32x4 o[NB][CT];
  float m_ref[NB], l_run[NB];

  // ---- the tile that starts at key kb, from its stage, which is refilled as soon
  // as it is free; every row sees the keys before `seen`
  auto tile = [&](Stage& st, int kb, int seen) __attribute__((always_inline)) {
    // V into LDS.  A token that is not a number counts through K (its score is
    // one for the rows that see it); its V becomes 0, so that no other row
    // takes it in with a weight of 0.
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float sv = mx_scale(st.sv[p] == kMxNan ? 0u : st.sv[p]);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const int chunk = qd * KS + i;           // 8 columns
        *reinterpret_cast<u32x4*>(vs + (p * 16 + l16) * D + ((chunk ^ swz_mx<D>(l16)) << 3)) =
            __builtin_bit_cast(u32x4, mx_values(st.v[p][i], sv));
      }
    }
    f32x4 s[NB][2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float sk = mx_scale(st.sk[p]);
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b][p] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const bf16x8 kf = mx_values(st.k[p][kk], sk);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            s[b][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qreg[b][kk][t], s[b][p], 0, 0, 0);
      }
    }
    load_tile(st);
    if (kb + kTK > seen) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (kb + 16 * p + 4 * qd + e > (STEP ? seen - 1 : lim[b])) s[b][p][e] = -INFINITY;
    }
    bf16x8 pb[NB][NT];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float mx = s[b][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[b][e >> 2][e & 3]);
      const float mxc = quad_max(mx) * c;
      const float m_new = (mxc > m_ref[b] + kRescaleSlack) ? mxc : m_ref[b];
      const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m_ref[b] - m_new);
      m_ref[b] = m_new;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[b][ct] *= alpha;
      }
      const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
      float pr[8], rs = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pr[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e >> 2][e & 3], c, -m_use));
        rs += pr[e];
      }
      l_run[b] = l_run[b] * alpha + rs;
      prob_terms(pr, pb[b]);
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      bf16x4 v[2];
#pragma unroll
      for (int p = 0; p < 2; ++p)
        v[p] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (lds_bf16x4*)(vl + p * 16 * D + vrow + (((2 * ct + vsub) ^ vswz) << 3)));
      const bf16x8 vf = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          o[b][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[b][t], o[b][ct], 0, 0, 0);
    }
  };

  // ---- the sequences of this slot.  Two tiles are in flight, and every step
  // issues the loads of one (past the wave's last tile they bring a tile again:
  // with a branch around them the compiler waits for all loads at every step).
  // `odd`: the next tile is in st[1].
  Stage st[2];
  page_ids();
  load_tile(st[0]);
  load_tile(st[1]);
  load_rows(si);
  bool odd = false, merged = false;
  for (; from < to; ++si) {
  const SeqDesc sd = a.seq[si];
  const int begin = a.tile_begin[si], end = a.tile_begin[si + 1];
  const int split = share == 0 ? 0 : unit - begin / share;
  const int nsplit = share == 0 ? 1 : (end - 1) / share - begin / share + 1;
  const int j0 = from - begin, j1 = min(to, end) - begin;
  from = begin + j1;
  const int rows = min(NB * 16, (STEP ? G : sd.suffix * G) - r0);
  if (!STEP && rows <= 0) {                               // chunks past this sequence's rows
    if (from < to) load_rows(si + 1);
    continue;
  }
  const int seen = sd.prefix + (STEP ? 0 : r0 / G) + 1;   // keys of the first row
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    m_ref[b] = -INFINITY, l_run[b] = 0.f;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) o[b][ct] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  int j = j0 + wave;
  if (odd && j < j1) {
    tile(st[1], j * kTK, seen);
    j += kWaves;
    odd = false;
  }
  for (; j + kWaves < j1; j += 2 * kWaves) {
    tile(st[0], j * kTK, seen);
    tile(st[1], (j + kWaves) * kTK, seen);
  }
  if (j < j1) {
    tile(st[0], j * kTK, seen);
    odd = true;
  }
  if (from < to) load_rows(si + 1);              // in flight during the merge

  // ---- merge the four waves.  Each parks its O rows in its own slot (its reads
  // of V precede these writes in LDS order), four columns a piece, the pieces of
  // a row XOR-swizzled by the row.
  constexpr int Q4 = D / 4;
  f32x4* ow = ring[wave].rows();
  if (MxDecSlot<D, NB>::kApart && merged) __syncthreads();   // the rows of the sequence before are read
  merged = true;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const float l_tot = quad_sum(l_run[b]);
    const int row = b * 16 + l16;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) ow[row * Q4 + ((ct * 4 + qd) ^ l16)] = o[b][ct];
    if (qd == 0) {
      ml[wave][row][0] = m_ref[b];
      ml[wave][row][1] = l_tot;
    }
  }
  __syncthreads();
  for (int idx = tid; idx < rows * Q4; idx += kWaves * 64) {
    const int r = idx / Q4, q = idx - r * Q4;
    float mstar = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mstar = fmaxf(mstar, ml[w][r][0]);
    float lsum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mw = ml[w][r][0];
      // a wave without tiles has m = -inf, l = 0 and O = 0; one whose scores
      // are all NaN has m = -inf too, and its l is NaN
      const float wt = (mw == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(mw - mstar);
      lsum += wt * ml[w][r][1];
      acc += wt * ring[w].rows()[r * Q4 + (q ^ (r & 15))];
    }
    const unsigned t = STEP ? 0u : (unsigned)(r0 + r) / (unsigned)G;
    const int local = (int)t * a.num_q_heads + g * G + (r0 + r - (int)t * G);   // row of the sequence
    if (nsplit == 1) {
      const int64_t row = (int64_t)sd.row_off * a.num_q_heads + local;
      const float inv = 1.0f / lsum;
      store4(reinterpret_cast<T*>(a.out) + row * D + q * 4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      if (a.lse != nullptr && q == 0) a.lse[row] = (mstar + __builtin_log2f(lsum)) * kLn2;
    } else {
      const int64_t prow = a.part_row[si] + (int64_t)split * sd.suffix * a.num_q_heads + local;
      *reinterpret_cast<f32x4*>(a.part_o + prow * D + q * 4) = acc;
      if (q == 0) *reinterpret_cast<f32x2*>(a.part_ml + prow * 2) = (f32x2){mstar, lsum};
    }
  }
  if (!MxDecSlot<D, NB>::kApart && from < to) __syncthreads();   // the slots are free again
  }
}

// The partial results of a row, in the order of its keys:
//   m* = max_s m_s,  w_s = 2^(m_s - m*),  out = sum_s w_s O_s / sum_s w_s l_s.
// D/4 lanes take a row's columns, four each; a workgroup's groups of such lanes
// share one row's partials (WIDE: a call with few rows and many partials is
// bound by memory round trips) or have a row each.
template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(256) void mx_join_kernel(const MxJoinArgs a) {
  constexpr int Q4 = D / 4, GROUPS = 256 / Q4, AHEAD = 8;
  __shared__ f32x4 part[WIDE ? GROUPS : 1][Q4];
  __shared__ float sums[WIDE ? GROUPS : 1];
  const int q = threadIdx.x % Q4, group = threadIdx.x / Q4;
  const int64_t at = WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * GROUPS + group;
  const bool live = at < a.row_begin[a.nseq];
  const int x = live ? (int)at : 0;
  const int si = find_seq(a.row_begin, a.nseq, x), h = x - a.row_begin[si];
  const int n = a.parts[si];
  const int64_t first = a.part_row[si] + h;
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml) + first;
  const f32x4* po = reinterpret_cast<const f32x4*>(a.part_o + first * D) + q;
  const int64_t step = a.row_begin[si + 1] - a.row_begin[si];
  float mstar = -INFINITY;
  for (int s = q; s < n; s += Q4) mstar = fmaxf(mstar, ml[s * step][0]);
#pragma unroll
  for (int d = Q4 / 2; d > 0; d >>= 1) mstar = fmaxf(mstar, __shfl_xor(mstar, d));
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float lsum = 0.f;
  constexpr int BY = WIDE ? GROUPS : 1;
  for (int s0 = WIDE ? group : 0; s0 < n; s0 += BY * AHEAD) {
    f32x4 v[AHEAD];
    f32x2 e[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (s0 + i * BY < n) v[i] = po[(s0 + i * BY) * step * Q4], e[i] = ml[(s0 + i * BY) * step];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (s0 + i * BY < n) {
        const float w = e[i][0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(e[i][0] - mstar);   // -inf: no keys, l and O 0
        lsum += w * e[i][1];
        acc += w * v[i];
      }
  }
  if constexpr (WIDE) {
    part[group][q] = acc;
    if (q == 0) sums[group] = lsum;
    __syncthreads();
    if (group != 0) return;
    acc = (f32x4){0.f, 0.f, 0.f, 0.f}, lsum = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) acc += part[i][q], lsum += sums[i];
  }
  if (!live) return;
  const int64_t row = (int64_t)a.row[si] + h;
  const float inv = 1.0f / lsum;
  store4(reinterpret_cast<T*>(a.out) + row * D + q * 4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  if (a.lse != nullptr && q == 0) a.lse[row] = (mstar + __builtin_log2f(lsum)) * kLn2;
}

template <typename T, int D>
void launch_join_as(const MxJoinArgs& a, hipStream_t stream) {
  const int64_t rows = a.row_begin[a.nseq], groups = 256 / (D / 4);
  if (rows < 4096)
    hipLaunchKernelGGL((mx_join_kernel<T, D, true>), dim3((unsigned)rows), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((mx_join_kernel<T, D, false>), dim3((unsigned)((rows + groups - 1) / groups)), dim3(256), 0,
                       stream, a);
}

template <typename T, int D>
void launch_as(const MxDecodeArgs& a, int grid, hipStream_t stream) {
  int most = 0, longest = 0;
  for (int i = 0; i < a.nseq; ++i) {
    longest = a.seq[i].suffix > longest ? a.seq[i].suffix : longest;
    most = a.seq[i].suffix * a.group > most ? a.seq[i].suffix * a.group : most;
  }
  const dim3 g(grid), b(kWaves * 64);
  if (longest == 1 && most <= 16) hipLaunchKernelGGL((mx_decode_kernel<T, D, 1, true>), g, b, 0, stream, a);
  else if (longest == 1) hipLaunchKernelGGL((mx_decode_kernel<T, D, 2, true>), g, b, 0, stream, a);
  else if (most <= 16) hipLaunchKernelGGL((mx_decode_kernel<T, D, 1, false>), g, b, 0, stream, a);
  else hipLaunchKernelGGL((mx_decode_kernel<T, D, 2, false>), g, b, 0, stream, a);
}

}  // namespace

hipError_t launch_mx_decode(const MxDecodeArgs& a, int dtype, int head_dim, int grid, hipStream_t stream) {
  if (dtype == 0 && head_dim == 128) launch_as<__bf16, 128>(a, grid, stream);
  else if (dtype == 0 && head_dim == 64) launch_as<__bf16, 64>(a, grid, stream);
  else if (dtype == 1 && head_dim == 128) launch_as<float, 128>(a, grid, stream);
  else launch_as<float, 64>(a, grid, stream);
  return hipGetLastError();
}

hipError_t launch_mx_join(const MxJoinArgs& a, int dtype, int head_dim, hipStream_t stream) {
  if (dtype == 0 && head_dim == 128) launch_join_as<__bf16, 128>(a, stream);
  else if (dtype == 0 && head_dim == 64) launch_join_as<__bf16, 64>(a, stream);
  else if (dtype == 1 && head_dim == 128) launch_join_as<float, 128>(a, stream);
  else launch_join_as<float, 64>(a, stream);
  return hipGetLastError();
}

}  // namespace kvt
