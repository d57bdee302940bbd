// Device-side helpers of 4-bit pages and of products that keep fp32 inputs
// (gfx950).
#pragma once

#include "kvt_device.h"
#include "kvt_mx.h"

namespace kvt {
namespace dev {

constexpr unsigned kMxNan = 255;   // scale byte of a token whose row holds an infinity or a NaN

// 2^(byte - 127); byte 255 makes every value that it scales a NaN (the
// conversion takes the scale's exponent bits, all ones, for that).
__device__ __forceinline__ float mx_scale(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// 8 codes as bf16, lowest nibble first: a code has 2 significant bits and the
// scale is a power of two, so every value is exact (scales of 2^-125 .. 2^96
// keep it normal).
__device__ __forceinline__ bf16x8 mx_values(unsigned codes, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}

// Unit and head of workgroup b of n = units * heads.  Workgroups go to the 8 XCDs
// in turn: all heads of a unit to one, 8 units at a time, so that its L2 holds the
// pages of a unit's tokens, where neighbouring records share lines (64 contexts of
// 1024..16384 keys, 8 kv-heads of 128: 445 -> 421 MB read, of 64 248 -> 209, and
// 84.9 -> 83.0 us, 58.8 -> 57.2).
struct Place8 {
  int unit, head;
};
__device__ __forceinline__ Place8 place_of(int b, int n, int heads) {
  const int group = b / (8 * heads), first = group * 8 * heads;
  const int width = min(8, (n - first) / heads);
  const int in = b - first;
  return {group * 8 + in % width, in / width};
}

// Terms of an element of T as bf16 numbers: bf16 is one, an fp32 number the sum
// of three (8 + 8 + 8 significant bits; the rest is under 2^-24 of it, and
// under 2^-133 where the terms reach the end of bf16's range).
template <typename T>
constexpr int kTerms = sizeof(T) == 2 ? 1 : 3;

__device__ __forceinline__ void split3(f32x4 a, f32x4 b, bf16x8 (&t)[3]) {
  const u32x4 hi = round8(a, b);
  auto rest = [](f32x4 x, unsigned p, unsigned q) __attribute__((always_inline)) {
    return (f32x4){x[0] - __builtin_bit_cast(float, p << 16), x[1] - __builtin_bit_cast(float, p & 0xffff0000u),
                   x[2] - __builtin_bit_cast(float, q << 16), x[3] - __builtin_bit_cast(float, q & 0xffff0000u)};
  };
  const f32x4 a1 = rest(a, hi[0], hi[1]), b1 = rest(b, hi[2], hi[3]);
  const u32x4 mid = round8(a1, b1);
  const u32x4 lo = round8(rest(a1, mid[0], mid[1]), rest(b1, mid[2], mid[3]));
  t[0] = __builtin_bit_cast(bf16x8, hi);
  t[1] = __builtin_bit_cast(bf16x8, mid);
  t[2] = __builtin_bit_cast(bf16x8, lo);
}

// 8 consecutive elements as the terms of their type.
__device__ __forceinline__ void load_terms(const __bf16* p, bf16x8 (&t)[1]) {
  t[0] = __builtin_bit_cast(bf16x8, load8(p));
}
__device__ __forceinline__ void load_terms(const float* p, bf16x8 (&t)[1]) {   // rounded
  t[0] = __builtin_bit_cast(bf16x8, load8(p));
}
__device__ __forceinline__ void load_terms(const float* p, bf16x8 (&t)[3]) {
  split3(*reinterpret_cast<const f32x4*>(p), *reinterpret_cast<const f32x4*>(p + 4), t);
}

// 8 probabilities (positive) as the terms of the storage type's precision.  bf16: one
// number, as the attention calls over bf16 pages have it.  The result is then off by
// 2.3e-3 (2-norm), 1.7e-3 of which are its own rounding; two numbers would leave
// those alone, for a second value product: 512 new tokens over 8192, 32/8 heads of
// 128, 81.3 -> 100.7 us, 2048 over 131072 3.82 -> 5.07 ms; a decoding step over one
// context of 131072 31.7 -> 32.5 us, over 64 of 1024..16384 82.2 -> 84.1.
__device__ __forceinline__ void prob_terms(const float (&p)[8], bf16x8 (&t)[1]) {
  t[0] = __builtin_bit_cast(bf16x8, round8((f32x4){p[0], p[1], p[2], p[3]}, (f32x4){p[4], p[5], p[6], p[7]}));
}
__device__ __forceinline__ void prob_terms(const float (&p)[8], bf16x8 (&t)[3]) {
  split3((f32x4){p[0], p[1], p[2], p[3]}, (f32x4){p[4], p[5], p[6], p[7]}, t);
}

// Own value and the one of lane l ^ 16 (v_permlane16_swap of x with itself
// leaves the even rows' values in the first result, the odd rows' in the second).
__device__ __forceinline__ void row_values(float x, float& a, float& b) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const unsigned p0 = p[0];
  const unsigned p1 = p[1];
  a = __builtin_bit_cast(float, p0);
  b = __builtin_bit_cast(float, p1);
}
// Maximum and sum over the four lanes l % 16 + {0, 16, 32, 48}.
__device__ __forceinline__ float quad_max(float x) {
  float a, b;
  row_values(x, a, b);
  return pair_max(fmaxf(a, b));
}
__device__ __forceinline__ float quad_sum(float x) {
  float a, b;
  row_values(x, a, b);
  return pair_sum(a + b);
}

}  // namespace dev
}  // namespace kvt
