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

// y of differential attention from both maps' unnormalised outputs.  Each
// product is rounded by itself: equal maps with lambda = 1 then cancel exactly,
// where a fused product would leave its own last bits.
__device__ __forceinline__ float map_difference(float o0, float inv0, float o1, float inv1, float lambda) {
#pragma clang fp contract(off)
  return o0 * inv0 - lambda * (o1 * inv1);
}

}  // namespace dev
}  // namespace kvt
