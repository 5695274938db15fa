// Eight elements at a time, values on their way to 8 bits, and a launch's status: shared by the kernels that write to the
// block cache.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.h"

namespace scoot {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
template <typename T>
struct Vec8;
template <>
struct Vec8<_Float16> {
  typedef h8 type;
};
template <>
struct Vec8<__bf16> {
  typedef b8 type;
};

// Not above the largest finite 8-bit float (e4m3); NaN stays NaN.
__device__ __forceinline__ float limited_f8(float x) { return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x; }
// What the nearest 8-bit float of x / scale is made of.
__device__ __forceinline__ float limit_f8(float x, float scale) { return limited_f8(x / scale); }

// Eight floats in range as 8-bit ones.
__device__ __forceinline__ int2 to_f8(const float (&f)[8]) {
  int w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j], f[4 * j + 1], 0, false);
    w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2], f[4 * j + 3], w[j], true);
  }
  return make_int2(w[0], w[1]);
}

inline int launched(const char* what) {
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return fail(SCOOT_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(err));
  return SCOOT_OK;
}

}  // namespace scoot
