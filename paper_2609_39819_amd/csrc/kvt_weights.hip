// Attention weight of every cached position, gfx950.
//
//   w[b][g][j] (+)= sum over the new rows (token i, head h of kv-head g) that
//                   see j of exp(scale <q_i,h, K_j> - lse_i,h)
// with the log-sum-exp that the attention call returned: half of its products,
// K once and no V.  Every weight is summed by one workgroup in a fixed order.
// Scores are fp32 sums of exact products: bf16 and 4-bit keys are bf16
// operands; fp32 ones three bf16 terms, whose products with a query's three
// are the six that reach 2^-24.  The log-sum-exp of the plain attention calls over
// fp32 pages is that of operands rounded to bf16, and weights that go with it need
// the same scores (kRounded).  8/2 heads over 4000 keys, scores spread over tens:
// rows add up to 1 within 1e-4 so, of the six products within 5e-2.
//
// Two kernels, by the rows that the largest sequence adds:
//   * step (at most 32 rows, a decoding step): HBM-bound on K.  4 waves stream
//     32-key tiles from HBM into their operands (no LDS), 16 or 32 rows by
//     v_mfma_f32_16x16x32_bf16, whose result holds four rows' scores of a key in a
//     lane: most of a key's sum is in the lane (with the keys' scores of a row in a
//     lane instead, 48 contexts took 42.8 us).  The batch's tiles lie one after the
//     other and every workgroup takes an equal share, of as many sequences as lie
//     there.  48 contexts of 1024..16384 keys over 4-bit pages, 32/8 heads of 128:
//     37.2 us; one of 131000 over bf16 pages 54.6 us (5.1 TB/s);
//   * turn: bound by the products and the exponentials (16 cycles of a wave's vector
//     unit for 64 of them, 8 more for a score's product and sum).  Every wave holds 32
//     keys as operands in registers; the rows pass through LDS, 256 in bf16 or 64
//     in fp32 at a time, two such stages in turn, for all waves of the workgroup.
//     512 new tokens over 8192, 32/8 heads of 128: 54.5 us, of which a full round of
//     wide workgroups is 39 (880 TFLOP/s) and a narrow one 15; fp32 192, rounded 91.
//     Vector instructions take 49 % of the SIMDs' cycles, products 28 %.
#include <type_traits>

#include "kvt_mx_device.h"

namespace kvt {
namespace {

using namespace dev;

template <int FORMAT>
constexpr int kKeyTerms = FORMAT == 1 ? 3 : 1;
template <typename T, int FORMAT>
constexpr int kQueryTerms = FORMAT == kRounded ? 1 : kTerms<T>;

// 8 fp32 columns of a key as its terms.
__device__ __forceinline__ void key_terms(u32x4 a, u32x4 b, bf16x8 (&t)[1]) {
  t[0] = __builtin_bit_cast(bf16x8, round8(__builtin_bit_cast(f32x4, a), __builtin_bit_cast(f32x4, b)));
}
__device__ __forceinline__ void key_terms(u32x4 a, u32x4 b, bf16x8 (&t)[3]) {
  split3(__builtin_bit_cast(f32x4, a), __builtin_bit_cast(f32x4, b), t);
}

// s += Q K^T (a lane has a key's scores of four rows), or K Q^T, over the terms of
// both whose product counts
template <int KN, int QN>
__device__ __forceinline__ void products16(f32x4& s, const bf16x8 (&k)[KN], const bf16x8 (&q)[QN]) {
#pragma unroll
  for (int i = 0; i < KN; ++i)
#pragma unroll
    for (int j = 0; j < QN; ++j)
      if (i + j < 3) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[j], k[i], s, 0, 0, 0);
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

// R: rows at most, 4, 8, 16 or 32.  A lane's four scores of a key are rows 4 qd ..
// of 16 (twice with 32).  Up to 8 rows are there more than once, so that a lane
// takes the exponentials of one of a tile's two pages only, and fewer lanes have
// to add up a key's sum.
template <typename T, int D, int FORMAT, int R>
__global__ __launch_bounds__(256, 2) void weights_step_kernel(const WeightsArgs a) {
  constexpr bool kCodes = FORMAT == kMx;
  constexpr int QN = kQueryTerms<T, FORMAT>, KN = kKeyTerms<FORMAT>;
  constexpr int KS = D / 32;
  constexpr int NB = R == 32 ? 2 : 1;
  constexpr bool kOnePage = R <= 8;              // of a tile, for each lane: page `half`
  constexpr int kTK = 32;
  constexpr int kPieces = kCodes ? 1 : FORMAT == 0 ? KS : 2 * KS;   // 16-byte loads per page and lane
  constexpr int64_t kPage = kCodes ? mx_page_bytes(D) : (int64_t)kBlock * D * (FORMAT == 0 ? 2 : 4);
  constexpr int DEPTH = FORMAT == 1 ? 1 : 2;     // tiles in flight
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, qd = lane >> 4;
  const int half = R == 8 ? qd >> 1 : qd & 1;    // the page whose weights this lane ends up with ...
  const bool writes = R == 8 ? (qd & 1) == 0 : qd < 2;   // ... and puts into place, key l16 of it
  const int mine = 16 * half + l16;

  const int hkv = a.num_kv_heads, G = a.group;
  // neighbouring records of 4-bit pages share lines: one XCD for all heads of a share
  // (37.7 -> 37.2 us; bf16 pages 54.6 -> 55.7, there a kv-head has an XCD)
  const Place8 at8 = kCodes ? place_of(blockIdx.x, gridDim.x, hkv)
                            : Place8{(int)(blockIdx.x / hkv), (int)(blockIdx.x % hkv)};
  const int g = at8.head;
  const char* kpool = reinterpret_cast<const char*>(a.k_pool);
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
  int from = at8.unit * a.share;
  const int to = min(from + a.share, a.unit_begin[a.nseq]);
  for (int si = find_seq(a.unit_begin, a.nseq, from); from < to; ++si) {   // the sequences of this slot
  const SeqDesc sd = a.seq[si];
  const int P = sd.prefix, L = P + sd.suffix, rows = sd.suffix * G;
  const int nblk = (L + kBlock - 1) / kBlock;
  const int j0 = from - a.unit_begin[si], j1 = min(to, a.unit_begin[si + 1]) - a.unit_begin[si];
  from = a.unit_begin[si] + j1;
  const int nt = j1 - j0 > wave ? (j1 - j0 - wave + 3) / 4 : 0;

  // ---- the query rows: this lane's operand is row l16 (% R) of 16, its scores are
  // those of rows 4 qd + e (% R).  A row past the last sees nothing.
  bf16x8 qreg[NB][KS][QN];
  float lse2[NB][4];
  int lim[NB][4];
  auto row_at = [&](int r, int& tok) __attribute__((always_inline)) {
    r = min(r, rows - 1);
    tok = r / G;
    return (int64_t)(sd.row_off + tok) * a.num_q_heads + g * G + (r - tok * G);
  };
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    int tok;
    const T* qp = reinterpret_cast<const T*>(a.q) + row_at(b * 16 + l16 % min(R, 16), tok) * D;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) load_terms(qp + (kCodes ? qd * (D / 4) + kk * 8 : kk * 32 + qd * 8), qreg[b][kk]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = b * 16 + (4 * qd + e) % min(R, 16);
      const float lse = a.lse[row_at(r, tok)];
      // a row past the last: 2^(s - infinity) = 0 (or NaN for a key that is one
      // anyway)
      lse2[b][e] = r < rows ? lse * kLog2e : INFINITY;
      lim[b][e] = P + tok;
    }
  }
  float* w = a.weights + ((int64_t)sd.seq * hkv + g) * a.stride;
  const __attribute__((address_space(4))) int32_t* bt =
      (const __attribute__((address_space(4))) int32_t*)(a.block_table + (int64_t)sd.seq * a.max_blocks);
  auto page_ids = [&](int j, uint32_t (&ids)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = __builtin_amdgcn_readfirstlane(min(j * 2 + p, nblk - 1));
      ids[p] = (uint32_t)bt[page];
    }
  };
  // (and the old weight of this lane's key, or else any 4 readable bytes)
  const float* old = P >= 1 ? w : reinterpret_cast<const float*>(a.q);
  struct Stage {
    u32x4 k[2][kPieces];
    unsigned char scale[2];
    float old;
  };
  auto load_tile = [&](int j, const uint32_t (&ids)[2], Stage& st) __attribute__((always_inline)) {
    st.old = old[max(0, min(j * kTK + mine, P - 1))];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int page = min(j * 2 + p, nblk - 1);
      const int slot = min(l16, L - 1 - page * kBlock);
      const char* at = kpool + ((int64_t)min(ids[p], nb_max) * hkv + g) * kPage;
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
    const float before = st.old;
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
        else key_terms(st.k[p][2 * kk], st.k[p][2 * kk + 1], kf);
#pragma unroll
        for (int b = 0; b < NB; ++b) products16(s[b][p], kf, qreg[b][kk]);
      }
    }
    next();
    auto sum_of = [&](auto masked) __attribute__((always_inline)) {
      auto p_of = [&](float x, int b, int e, int key) __attribute__((always_inline)) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, c, -lse2[b][e]));
        return decltype(masked)::value && key > lim[b][e] ? 0.f : p;
      };
      if constexpr (kOnePage) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += p_of(half ? s[0][1][e] : s[0][0][e], 0, e, kb + mine);
        if constexpr (R == 8) {                  // rows 0..3 here, 4..7 in lane l ^ 16
          float x, y;
          row_values(sum, x, y);
          sum = x + y;
        }
        return sum;
      } else {
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[p] += p_of(s[b][p][e], b, e, kb + 16 * p + l16);
        // lanes of even 16s keep page 0's and odd ones page 1's, of four rows here and four there
        const auto both = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, sum[0]),
                                                           __builtin_bit_cast(unsigned, sum[1]), false, false);
        const unsigned x = both[0], y = both[1];
        return pair_sum(__builtin_bit_cast(float, x) + __builtin_bit_cast(float, y));
      }
    };
    const int key = kb + mine;
    if (kb + kTK <= P) {                         // every row sees all of the tile, every key has an old weight
      const float sum = sum_of(std::false_type());
      if (writes) w[key] = before + sum;
    } else {
      const float sum = sum_of(std::true_type());
      if (writes && key < L) w[key] = key < P ? before + sum : sum;
    }
  };

  // past the last tile the loads bring it again: every step issues as many
  auto jt = [&](int i) { return j0 + wave + 4 * min(i, nt - 1); };
  Stage st[DEPTH];
  uint32_t ids[2];
  if (nt > 0) {
    page_ids(jt(0), ids);
#pragma unroll
    for (int x = 0; x < DEPTH; ++x) {
      load_tile(jt(x), ids, st[x]);
      page_ids(jt(x + 1), ids);
    }
    auto step = [&](int i, Stage& s) __attribute__((always_inline)) {
      tile(s, jt(i) * kTK, [&]() __attribute__((always_inline)) {
        load_tile(jt(i + DEPTH), ids, s);
        page_ids(jt(i + DEPTH + 1), ids);
      });
    };
    int i = 0;
    for (; i + DEPTH <= nt; i += DEPTH)
#pragma unroll
      for (int x = 0; x < DEPTH; ++x) step(i + x, st[x]);
    if (i < nt) step(i, st[0]);
  }
  }
}

// Rows of queries in LDS at a time, as the operand terms of their type: [term][row][D] bf16,
// the 16-byte chunks of a row XOR-swizzled as a key tile's in the extend kernel.
template <typename T>
constexpr int kTurnRows = weights_stage_rows(sizeof(T) == 2 ? 0 : 1);
template <typename T, int D, int QN>
struct TurnRows {
  __bf16 q[QN][kTurnRows<T> * D];
  float lse[kTurnRows<T>];
  int lim[kTurnRows<T>];
};

template <typename T, int D, int FORMAT, bool ONCE>
__global__ __launch_bounds__(512) void weights_turn_kernel(const WeightsArgs a) {
  constexpr bool kCodes = FORMAT == kMx;
  constexpr bool kDirect = sizeof(T) == 2;       // rows go straight into LDS
  constexpr int QN = kQueryTerms<T, FORMAT>, KN = kKeyTerms<FORMAT>;
  constexpr int KSTEPS = D / 16, CHUNKS = D / 8;
  constexpr int ROWS = kTurnRows<T>, BLOCKS = ROWS / 32;
  static_assert(!kDirect || BLOCKS == 8, "a narrow workgroup's waves have a block each");
  typedef TurnRows<T, D, QN> Rows;
  constexpr int64_t kPage = kCodes ? mx_page_bytes(D) : (int64_t)kBlock * D * (FORMAT == 0 ? 2 : 4);
  constexpr int PIECES = ROWS * CHUNKS / 512;    // of 8 columns, per thread and stage
  extern __shared__ __attribute__((aligned(1024))) char turn_lds[];
  Rows* stage = reinterpret_cast<Rows*>(turn_lds);   // two
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, l32 = lane & 31;

  // ---- a wide workgroup has 32 keys per wave and every wave takes all rows, a
  // narrow one has 32 keys and its waves take the blocks of 32 rows in turn.  ONCE: the
  // rows of every sequence are one stage, which stays in LDS, and a workgroup (all
  // are wide) goes through a.tiles tiles of keys, the next one's in flight.
  const int hkv = a.num_kv_heads, G = a.group;
  const int g = blockIdx.x % hkv;
  const int unit = blockIdx.x / hkv;
  const bool narrow = !ONCE && unit >= a.unit_begin[a.nseq];
  const int at = narrow ? unit - a.unit_begin[a.nseq] : unit;
  const int si = find_seq(narrow ? a.narrow_begin : a.unit_begin, a.nseq, at);
  const SeqDesc sd = a.seq[si];
  const int P = sd.prefix, L = P + sd.suffix, rows = sd.suffix * G;
  const int stages = (rows + ROWS - 1) / ROWS;
  const int step = narrow ? 32 : kWeightsWideKeys;       // keys of a tile
  const int wide_keys = (a.unit_begin[si + 1] - a.unit_begin[si]) * kWeightsWideKeys;   // where there are narrow ones
  const int start = narrow ? wide_keys + (at - a.narrow_begin[si]) * 32
                           : (at - a.unit_begin[si]) * kWeightsWideKeys * (ONCE ? a.tiles : 1);
  const int stop = start + (ONCE ? min(L - start, a.tiles * kWeightsWideKeys) : step);
  const int nblk = (L + kBlock - 1) / kBlock;
  float* w = a.weights + ((int64_t)sd.seq * hkv + g) * a.stride;

  // ---- the keys from kb on, one a lane pair, as stored (past the end the last
  // one: not stored)
  const uint32_t nb_max = (uint32_t)min<int64_t>(a.num_blocks, 0x7fffffff) - 1u;
  constexpr int KP = kCodes ? D / 64 : KSTEPS * (FORMAT == 0 ? 1 : 2);   // 16-byte pieces of a lane's columns
  constexpr bool kFly = ONCE && (kCodes || FORMAT == 0);   // the next tile's in flight (fp32: too many registers)
  u32x4 kraw[KP];
  unsigned char kscale[kCodes ? D / 64 : 1];
  auto page_of = [&](int kb) __attribute__((always_inline)) {
    const int pos = min(kb + l32, L - 1);
    return (uint32_t)a.block_table[(int64_t)sd.seq * a.max_blocks + min(pos / kBlock, nblk - 1)];
  };
  auto load_keys = [&](int kb, uint32_t id) __attribute__((always_inline)) {
    const int slot = min(kb + l32, L - 1) % kBlock;
    const char* page = reinterpret_cast<const char*>(a.k_pool) + ((int64_t)min(id, nb_max) * hkv + g) * kPage;
    if constexpr (kCodes) {
#pragma unroll
      for (int y = 0; y < KP; ++y) {             // 32 columns: four words under one scale
        kraw[y] = *reinterpret_cast<const u32x4*>(page + slot * (D / 2) + hh * (D / 4) + y * 16);
        kscale[y] = (unsigned char)page[mx_code_bytes(D) + slot * (D / 32) + hh * (D / 64) + y];
      }
    } else {
      constexpr int ES = FORMAT == 0 ? 2 : 4, PER = FORMAT == 0 ? 1 : 2;
#pragma unroll
      for (int y = 0; y < KP; ++y)
        kraw[y] = *reinterpret_cast<const u32x4*>(page + (slot * D + (y / PER) * 16 + hh * 8) * ES + 16 * (y % PER));
    }
  };
  bf16x8 kf[KSTEPS][KN];
  auto take_keys = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) {
      if constexpr (kCodes) kf[kk][0] = mx_values(kraw[kk / 4][kk % 4], mx_scale(kscale[kk / 4]));
      else if constexpr (FORMAT == 0) kf[kk][0] = __builtin_bit_cast(bf16x8, kraw[kk]);
      else key_terms(kraw[2 * kk], kraw[2 * kk + 1], kf[kk]);
    }
  };
  int kb = start + (narrow ? 0 : wave * 32);
  uint32_t id = page_of(kb);

  const float c = a.scale_log2;
  const int k32 = 8 * (l32 >> 3) + 4 * hh + (l32 >> 1 & 3);   // the key whose sum ends in this lane
  // the waves' sums of the keys from kb on, as scatter_sum leaves them
  auto join_waves = [&](float sum) __attribute__((always_inline)) {
    float* red = reinterpret_cast<float*>(turn_lds);   // the rows are done with
    __syncthreads();
    if ((lane & 1) == 0) red[wave * 32 + k32] = sum;
    __syncthreads();
    if (tid < 32 && kb + tid < L) {
      sum = 0.f;
      for (int x = 0; x < 8; ++x) sum += red[x * 32 + tid];
      put(w, kb + tid, sd, sum);
    }
  };
  if constexpr (!ONCE && !kDirect) {
    // a narrow workgroup's fp32 rows, each used once, go straight into operands: a
    // stage holds blocks for two of the waves only (512 new tokens over 8192, 32/8
    // heads of 128: 214 us by stages, 192 so, of 64 over 4-bit pages 91 and 59; bf16
    // rows, whose stages hold eight blocks, 54.5 and 61)
    if (narrow) {
      load_keys(kb, id);
      take_keys();
      float acc[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = 0.f;
      const int blocks = (rows + 31) / 32;
      const int seeing = start > P ? (int)((int64_t)(start - P) * G / 32) : 0;   // blocks before see none of the keys
      for (int block = seeing + wave; block < blocks; block += 8) {
        const unsigned x = (unsigned)block * 32u + (unsigned)l32, r = min(x, (unsigned)rows - 1u), tok = r / (unsigned)G;
        const int64_t row = (int64_t)(sd.row_off + (int)tok) * a.num_q_heads + g * G + (int)(r - tok * G);
        const T* q = reinterpret_cast<const T*>(a.q) + row * D;
        const float lse2 = a.lse[row] * kLog2e;
        const int thr = (x < (unsigned)rows ? P + (int)tok : -1) - kb - 4 * hh;    // keys past it: not seen
        f32x16 s = (f32x16){};
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) {
          bf16x8 qf[QN];
          load_terms(q + (kCodes ? hh * (D / 16) + kk : 2 * kk + hh) * 8, qf);
          products32(s, kf[kk], qf);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -lse2));
          acc[e] += 8 * (e >> 2) + (e & 3) > thr ? 0.f : p;
        }
      }
      const float sum = scatter_sum(acc, lane, 16);
      join_waves(sum + __shfl_xor(sum, 1));
      return;
    }
  }

  // ---- rows in stages, from the first that sees one of the workgroup's keys.
  // Row r of a stage whose first row is head h0 of token t0 is head x - d * G of
  // token t0 + d, d = x / G, x = h0 + r < G + ROWS.
  const int first = !ONCE && start > P ? (int)((int64_t)(start - P) * G / ROWS) : 0;
  const int adv_t = ROWS / G, adv_h = ROWS - adv_t * G;
  int t0 = (int)((int64_t)first * ROWS / G), h0 = first * ROWS - t0 * G;    // of the stage that is loaded next
  auto place = [&](int r, int& tok, int64_t& row) __attribute__((always_inline)) {
    const int x = h0 + r;
    const int d = G == 1 ? x : (int)(__umulhi((unsigned)x, a.by_group) >> a.group_shift);
    tok = t0 + d;
    const bool past = tok >= sd.suffix;          // past the last row: any row, it sees nothing
    row = (int64_t)(sd.row_off + (past ? 0 : tok)) * a.num_q_heads + g * G + (x - d * G);
  };
  constexpr int QP = (int)sizeof(T) / 2;
  u32x4 raw[kDirect ? 1 : PIECES][QP];
  float lse_raw = 0.f;
  int lim_raw = -1;
  // bf16 rows go straight into LDS: load i of a wave brings 64 pieces, and lane l
  // lands at piece l of them, so it fetches the chunk that the swizzle puts there;
  // fp32 rows pass through registers (drop), where they become their terms
  auto load_stage = [&](Rows& to) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < PIECES; ++x) {
      const int p = (kDirect ? (wave * PIECES + x) * 64 + lane : tid + x * 512);
      const int r = p / CHUNKS, chunk = kDirect ? (p % CHUNKS) ^ swz<D>(r) : p % CHUNKS;
      int tok;
      int64_t row;
      place(r, tok, row);
      const char* q = reinterpret_cast<const char*>(reinterpret_cast<const T*>(a.q) + row * D + chunk * 8);
      if constexpr (kDirect) {
        __builtin_amdgcn_global_load_lds(
            (const void*)q, (__attribute__((address_space(3))) void*)((lds_bf16*)to.q[0] + (wave * PIECES + x) * 512), 16,
            0, 0);
      } else {
#pragma unroll
        for (int y = 0; y < QP; ++y) raw[x][y] = *reinterpret_cast<const u32x4*>(q + 16 * y);
      }
    }
    if (tid < ROWS) {
      int tok;
      int64_t row;
      place(tid, tok, row);
      lse_raw = a.lse[row];
      lim_raw = tok >= sd.suffix ? -1 : P + tok;
    }
    t0 += adv_t;
    h0 += adv_h;
    if (h0 >= G) h0 -= G, ++t0;
  };
  auto drop = [&](Rows& to) __attribute__((always_inline)) {
    if constexpr (!kDirect) {
#pragma unroll
      for (int x = 0; x < PIECES; ++x) {
        const int p = tid + x * 512, r = p / CHUNKS, piece = r * D + (((p % CHUNKS) ^ swz<D>(r)) << 3);
        bf16x8 terms[QN];
        key_terms(raw[x][0], raw[x][1], terms);
#pragma unroll
        for (int y = 0; y < QN; ++y) *reinterpret_cast<u32x4*>(to.q[y] + piece) = __builtin_bit_cast(u32x4, terms[y]);
      }
    }
    if (tid < ROWS) to.lse[tid] = lse_raw, to.lim[tid] = lim_raw;
  };

  float acc[16];
  auto scores = [&](const Rows& from, int block) __attribute__((always_inline)) {
    const int row = block * 32 + l32;
    f32x16 s = (f32x16){};
#pragma unroll
    for (int kk = 0; kk < KSTEPS; ++kk) {
      const int chunk = kCodes ? hh * (D / 16) + kk : 2 * kk + hh;
      bf16x8 qf[QN];
#pragma unroll
      for (int y = 0; y < QN; ++y)
        qf[y] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(from.q[y] + row * D + ((chunk ^ swz<D>(l32)) << 3)));
      products32(s, kf[kk], qf);
    }
    return s;
  };
  auto add = [&](const Rows& from, int block, const f32x16& s, auto masked) __attribute__((always_inline)) {
    const float lse2 = from.lse[block * 32 + l32] * kLog2e;
    const int thr = decltype(masked)::value ? from.lim[block * 32 + l32] - kb - 4 * hh : 0;   // keys past lim: offset > thr
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -lse2));
      if constexpr (decltype(masked)::value) acc[e] += 8 * (e >> 2) + (e & 3) > thr ? 0.f : p;
      else acc[e] += p;
    }
  };
  // one stage of rows, the first of which is `seen`'s and sees the fewest keys
  auto take_rows = [&](const Rows& cur, int seen, int last) __attribute__((always_inline)) {
    if (kDirect && narrow) {
      add(cur, wave, scores(cur, wave), std::true_type());
    } else if (P + seen >= kb + 31 && last <= rows) {
      f32x16 s = scores(cur, 0);
#pragma unroll
      for (int block = 0; block < BLOCKS; ++block) {
        f32x16 s1 = s;
        if (block + 1 < BLOCKS) s1 = scores(cur, block + 1);
        add(cur, block, s, std::false_type());
        s = s1;
        if constexpr (QN == 1 && KN == 1) {      // the next products beside the exponentials
          __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
          for (int i = 0; i < KSTEPS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 48 / KSTEPS, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
        }
      }
    } else {
      const int blocks = min(BLOCKS, (rows - (last - ROWS) + 31) / 32);
      for (int block = 0; block < blocks; ++block) add(cur, block, scores(cur, block), std::true_type());
    }
  };
  int seen = t0, seen_h = h0;
  load_stage(stage[0]);
  load_keys(kb, id);
  drop(stage[0]);
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  __syncthreads();
  for (int base = start; base < stop; base += step) {
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    if (ONCE && !kFly && base != start) load_keys(kb, id);
    take_keys();
    const float old = w[min(kb + k32, L - 1)];
    const int next = kb + step;
    if constexpr (ONCE) {
      if (base + step < stop) {
        id = page_of(next);
        if (kFly) load_keys(next, id);
      }
      take_rows(stage[0], 0, ROWS);
    } else {
      for (int i = first; i < stages; ++i) {
        Rows& fill = stage[(i + 1 - first) & 1];
        if (i + 1 < stages) load_stage(fill);
        take_rows(stage[(i - first) & 1], seen, (i + 1) * ROWS);
        seen += adv_t;
        seen_h += adv_h;
        if (seen_h >= G) seen_h -= G, ++seen;
        if (i + 1 < stages) drop(fill);
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        __syncthreads();
      }
    }
    // ---- sums over the rows: the lanes of a half, and of a narrow workgroup the
    // waves, in order
    float sum = scatter_sum(acc, lane, 16);      // of element l32 >> 1, half of it
    sum += __shfl_xor(sum, 1);
    if (!narrow) {
      if ((lane & 1) == 0 && kb + k32 < L) w[kb + k32] = kb + k32 < P ? old + sum : sum;
    } else {
      join_waves(sum);
    }
    kb = next;
  }
}

template <typename T, int D, int FORMAT>
void launch_step_as(const WeightsArgs& a, int grid, hipStream_t stream) {
  int rows = 0;
  for (int i = 0; i < a.nseq; ++i) rows = a.seq[i].suffix * a.group > rows ? a.seq[i].suffix * a.group : rows;
  const dim3 g(grid), b(256);
  if (rows <= 4) hipLaunchKernelGGL((weights_step_kernel<T, D, FORMAT, 4>), g, b, 0, stream, a);
  else if (rows <= 8) hipLaunchKernelGGL((weights_step_kernel<T, D, FORMAT, 8>), g, b, 0, stream, a);
  else if (rows <= 16) hipLaunchKernelGGL((weights_step_kernel<T, D, FORMAT, 16>), g, b, 0, stream, a);
  else hipLaunchKernelGGL((weights_step_kernel<T, D, FORMAT, 32>), g, b, 0, stream, a);
}
template <typename T, int D, int FORMAT>
void launch_turn_as(const WeightsArgs& a, int grid, hipStream_t stream) {
  constexpr unsigned kStage = sizeof(TurnRows<T, D, kQueryTerms<T, FORMAT>>);
  if (a.tiles > 0)
    hipLaunchKernelGGL((weights_turn_kernel<T, D, FORMAT, true>), dim3(grid), dim3(512), kStage, stream, a);
  else
    hipLaunchKernelGGL((weights_turn_kernel<T, D, FORMAT, false>), dim3(grid), dim3(512), 2 * kStage, stream, a);
}

}  // namespace

hipError_t launch_weights_step(const WeightsArgs& a, int format, int dtype, int head_dim, int grid, hipStream_t stream) {
  const bool wide = head_dim == 128;
  if (format == 0) wide ? launch_step_as<__bf16, 128, 0>(a, grid, stream) : launch_step_as<__bf16, 64, 0>(a, grid, stream);
  else if (format == 1) wide ? launch_step_as<float, 128, 1>(a, grid, stream) : launch_step_as<float, 64, 1>(a, grid, stream);
  else if (format == kRounded) wide ? launch_step_as<float, 128, kRounded>(a, grid, stream) : launch_step_as<float, 64, kRounded>(a, grid, stream);
  else if (dtype == 0) wide ? launch_step_as<__bf16, 128, kMx>(a, grid, stream) : launch_step_as<__bf16, 64, kMx>(a, grid, stream);
  else wide ? launch_step_as<float, 128, kMx>(a, grid, stream) : launch_step_as<float, 64, kMx>(a, grid, stream);
  return hipGetLastError();
}

hipError_t launch_weights_turn(const WeightsArgs& a, int format, int dtype, int head_dim, int grid, hipStream_t stream) {
  const bool wide = head_dim == 128;
  if (format == 0) wide ? launch_turn_as<__bf16, 128, 0>(a, grid, stream) : launch_turn_as<__bf16, 64, 0>(a, grid, stream);
  else if (format == 1) wide ? launch_turn_as<float, 128, 1>(a, grid, stream) : launch_turn_as<float, 64, 1>(a, grid, stream);
  else if (format == kRounded) wide ? launch_turn_as<float, 128, kRounded>(a, grid, stream) : launch_turn_as<float, 64, kRounded>(a, grid, stream);
  else if (dtype == 0) wide ? launch_turn_as<__bf16, 128, kMx>(a, grid, stream) : launch_turn_as<__bf16, 64, kMx>(a, grid, stream);
  else wide ? launch_turn_as<float, 128, kMx>(a, grid, stream) : launch_turn_as<float, 64, kMx>(a, grid, stream);
  return hipGetLastError();
}

}  // namespace kvt
