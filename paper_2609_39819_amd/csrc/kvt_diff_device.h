// Device-side helpers of the differential attention kernels.
#pragma once

#include "kvt_device.h"
#include "kvt_diff.h"

namespace kvt {
namespace dev {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }

// A probability as two bf16 numbers: w is the probability cut off to bf16, the rest
// what is cut off and 2^-8 of the probability more, so that it is never 0 where w is
// not, and an infinite value times both stays one.  Together they are kOver times the
// probability (off by 2^-14 of it at most), which its sum is multiplied by in the end.
// Two probabilities at a time, packed.
constexpr float kOver = 1.0f + 0x1p-8f;
__device__ __forceinline__ void two_numbers(float p0, float p1, unsigned& w, unsigned& rest) {
  const unsigned u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
  const float r0 = __builtin_fmaf(p0, kOver, -__uint_as_float(u0 & 0xffff0000u));
  const float r1 = __builtin_fmaf(p1, kOver, -__uint_as_float(u1 & 0xffff0000u));
  w = __builtin_amdgcn_perm(u1, u0, 0x07060302u);   // both upper halves
  rest = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){r0, r1}, bf16x2));
}

// y of differential attention from both maps' unnormalised outputs.  Each
// product is rounded by itself: equal maps with lambda = 1 then cancel exactly,
// where a fused product would leave its own last bits.
__device__ __forceinline__ float map_difference(float o0, float inv0, float o1, float inv1, float lambda) {
#pragma clang fp contract(off)
  return o0 * inv0 - lambda * (o1 * inv1);
}

}  // namespace dev
}  // namespace kvt
