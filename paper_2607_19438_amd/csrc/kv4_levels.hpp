// The 4-bit cache's levels as bf16, for the kernels that read it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qgemm_kernels.hpp"

namespace qg {
namespace {

// Two levels of a packed byte (0..3 of w) times 2^(e-127); exact in bf16, NaN for e = 255.
template <int B>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float unit) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, B));
}

// Eight levels of a packed dword times 2^(e-127), as bf16.
__device__ __forceinline__ u32x4 fp4_unit(uint32_t w, float unit) {
  return u32x4{fp4_pair<0>(w, unit), fp4_pair<1>(w, unit), fp4_pair<2>(w, unit), fp4_pair<3>(w, unit)};
}

}  // namespace
}  // namespace qg
