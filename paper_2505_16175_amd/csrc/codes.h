// E4M3 codes of paged pools by the conversion instructions.
#pragma once
#include <hip/hip_runtime.h>

#include "append.h"

namespace qp {

// 4 f32 values as E4M3 codes: nearest, ties to even; what is beyond +-most saturates, NaN stays.
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float most = 448.f) {
  auto in = [=](float x) { return __builtin_elementwise_minimum(__builtin_elementwise_maximum(x, -most), most); };
  const unsigned lo = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), (int)lo, true);
}
// Four codes of values that are to be multiplied by a power of two (at most 1): exact down to the codes' subnormal values, rounded there.
__device__ __forceinline__ unsigned shrink4(unsigned w, float by) {
  return codes4(__builtin_amdgcn_cvt_f32_fp8(w, 0) * by, __builtin_amdgcn_cvt_f32_fp8(w, 1) * by, __builtin_amdgcn_cvt_f32_fp8(w, 2) * by,
                __builtin_amdgcn_cvt_f32_fp8(w, 3) * by);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }  // e from -126 to 127
// Exponent of a scale, whatever bits are there.
__device__ __forceinline__ int scale_exponent(float scale, int least, int most) {
  return min(max((int)((__float_as_uint(scale) >> 23) & 255u) - 127, least), most);
}

}  // namespace qp
