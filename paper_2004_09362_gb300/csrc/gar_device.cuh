// Element conversions and launch helpers shared by the decoding operators' kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <string>

#include "gar_internal.hpp"

namespace gar {

// An 8-bit float (4 exponent, 3 mantissa bits) and a signed 8-bit integer as storage.
struct e4m3 {
  uint8_t bits;
};
struct i8 {
  int8_t value;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(i8 x) { return (float)x.value; }
__device__ __forceinline__ float to_f32(e4m3 x) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)x.bits));
  return __half2float(__ushort_as_half((unsigned short)(h2 & 0xffff)));
}

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
// Quantised codes of x / scale, to the nearest, ties to even; |x / scale| is at most a
// rounding error over the type's largest value unless the scale is a subnormal.
template <> __device__ __forceinline__ i8 from_f32<i8>(float x) {
  return i8{(int8_t)__float2int_rn(fminf(fmaxf(x, -127.f), 127.f))};
}
template <> __device__ __forceinline__ e4m3 from_f32<e4m3>(float x) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
  return e4m3{(uint8_t)(r & 0xff)};
}

template <typename T> struct quantised {
  static constexpr bool value = false;
  static constexpr float largest = 1.f;
};
template <> struct quantised<i8> {
  static constexpr bool value = true;
  static constexpr float largest = 127.f;
};
template <> struct quantised<e4m3> {
  static constexpr bool value = true;
  static constexpr float largest = 448.f;
};

// N elements of T as one aligned access.
template <typename T, int N> struct alignas(sizeof(T) * N) pack {
  T e[N];
};

template <typename T> struct type_tag {
  using type = T;
};

inline bool float_type(int dtype) { return dtype == GAR_F32 || dtype == GAR_BF16 || dtype == GAR_F16; }
inline int element_size(int dtype) { return dtype == GAR_F32 ? 4 : dtype == GAR_I8 || dtype == GAR_E4M3 ? 1 : 2; }

// Calls f with the tag of the float type `dtype` (checked before).
template <typename F> int with_float(int dtype, F f) {
  if (dtype == GAR_F32) return f(type_tag<float>{});
  if (dtype == GAR_BF16) return f(type_tag<__nv_bfloat16>{});
  return f(type_tag<__half>{});
}

inline int launched(const char *what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? GAR_OK : cuda_fail(e, what);
}

inline int refuse(const std::string &why) {
  set_error(why);
  return GAR_EINVAL;
}

// cache.cu
int check_cache(const gar_kv_cache *cache);

}  // namespace gar
