// Folds over the 64 lanes of a wave on the VALU (DPP lane selects), and bf16 widening: shared by the gating kernels.
#pragma once
#include "common.h"

namespace moe {

template <int CTRL, int RMASK>
__device__ __forceinline__ float dpp_or(float keep, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(keep), __float_as_int(v), CTRL, RMASK, 0xF, false));
}
// Sum of the 64 lane values, pairing lanes at strides 1,2,4,8,16,32; every lane returns the total.
__device__ __forceinline__ float fold_sum(float a) {
  a = a + dpp_or<0xB1, 0xF>(0.0f, a);    // quad_perm [1,0,3,2]  : stride 1
  a = a + dpp_or<0x4E, 0xF>(0.0f, a);    // quad_perm [2,3,0,1]  : stride 2
  a = a + dpp_or<0x141, 0xF>(0.0f, a);   // row_half_mirror      : stride 4
  a = a + dpp_or<0x140, 0xF>(0.0f, a);   // row_mirror           : stride 8
  a = a + dpp_or<0x142, 0xA>(0.0f, a);   // row_bcast15 into rows 1 and 3 : stride 16
  a = a + dpp_or<0x143, 0xC>(0.0f, a);   // row_bcast31 into rows 2 and 3 : stride 32
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(a), 63));
}
__device__ __forceinline__ float fold_max(float a) {
  a = fmaxf(a, dpp_or<0xB1, 0xF>(a, a));
  a = fmaxf(a, dpp_or<0x4E, 0xF>(a, a));
  a = fmaxf(a, dpp_or<0x141, 0xF>(a, a));
  a = fmaxf(a, dpp_or<0x140, 0xF>(a, a));
  a = fmaxf(a, dpp_or<0x142, 0xA>(a, a));
  a = fmaxf(a, dpp_or<0x143, 0xC>(a, a));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(a), 63));
}

// Inclusive sum over the lanes of a wave
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // within rows of 16: from 1, 2, 4, 8 lanes before
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // a row's last lane to the next row
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // lane 31 to the upper half
  return v;
}

__device__ __forceinline__ void widen8(u32x4 v, float* f) {
  f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
  f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}

}  // namespace moe
