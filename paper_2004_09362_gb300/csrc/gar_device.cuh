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
// Two 32-bit operations in one instruction, each rounded as the single one.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{.reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mul.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x;}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{.reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x;}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{.reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 x, x, y, z; "
      "mov.b64 {%0, %1}, x;}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

// Four 8-bit codes of values within the type's range (a rounding error over it counts as within), to
// the nearest, ties to even.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, i8) {
  // Adding 1.5 * 2^23 rounds to an integer and leaves it in the low bits.
  const float2 big = make_float2(12582912.f, 12582912.f);
  const float2 ab = add2(make_float2(a, b), big), cd = add2(make_float2(c, d), big);
  return __byte_perm(__byte_perm(__float_as_uint(ab.x), __float_as_uint(ab.y), 0x0040),
                     __byte_perm(__float_as_uint(cd.x), __float_as_uint(cd.y), 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, e4m3) {
  uint16_t x, y;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(x) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(y) : "f"(d), "f"(c));
  return (uint32_t)x | (uint32_t)y << 16;
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

// 16 bytes of T as they lie in memory, and their values.  Held packed so that many can be in flight.
template <typename T> struct chunk16 {
  static constexpr int N = 16 / sizeof(T);
  uint4 bits;
};
__device__ __forceinline__ float2 unpack2(uint32_t x, __nv_bfloat16) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t x, __half) { return __half22float2(*reinterpret_cast<__half2 *>(&x)); }
// Four 8-bit codes' values.
__device__ __forceinline__ void unpack4(uint32_t x, float2 *ab, float2 *cd, i8) {
  // 0x4b000000 + u is 2^23 + u; with u = code + 128, taking away 2^23 + 128 leaves the code.
  const uint32_t u = x ^ 0x80808080u, e = 0x4b000000u;
  const float2 off = make_float2(-8388736.f, -8388736.f);
  *ab = add2(make_float2(__uint_as_float(__byte_perm(u, e, 0x7440)), __uint_as_float(__byte_perm(u, e, 0x7441))), off);
  *cd = add2(make_float2(__uint_as_float(__byte_perm(u, e, 0x7442)), __uint_as_float(__byte_perm(u, e, 0x7443))), off);
}
__device__ __forceinline__ void unpack4(uint32_t x, float2 *ab, float2 *cd, e4m3) {
  uint32_t l, h;
  asm("{.reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b;}" : "=r"(l), "=r"(h) : "r"(x));
  *ab = __half22float2(*reinterpret_cast<__half2 *>(&l));
  *cd = __half22float2(*reinterpret_cast<__half2 *>(&h));
}
__device__ __forceinline__ uint32_t pack2(float2 x, __nv_bfloat16) {
  const __nv_bfloat162 y = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t *>(&y);
}
__device__ __forceinline__ uint32_t pack2(float2 x, __half) {
  const __half2 y = __floats2half2_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t *>(&y);
}
template <typename T> __device__ __forceinline__ void unpack(const chunk16<T> &c, float (&v)[chunk16<T>::N]) {
  const uint32_t w[4] = {c.bits.x, c.bits.y, c.bits.z, c.bits.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      v[i] = __uint_as_float(w[i]);
    } else {
      const float2 x = unpack2(w[i], T());
      v[2 * i] = x.x, v[2 * i + 1] = x.y;
    }
  }
}
template <typename T> __device__ __forceinline__ chunk16<T> packed(const float (&v)[chunk16<T>::N]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4)
      w[i] = __float_as_uint(v[i]);
    else
      w[i] = pack2(make_float2(v[2 * i], v[2 * i + 1]), T());
  }
  return {make_uint4(w[0], w[1], w[2], w[3])};
}

// N (cos, sin) entries of a rotation table, 16 bytes a load where WIDE; NaN where `good` is false.
template <int N, bool WIDE>
__device__ __forceinline__ void load_rotation(const float2 *t, bool good, float (&c)[N], float (&s)[N]) {
  const float nan = __int_as_float(0x7fc00000);
  if (WIDE && N % 2 == 0) {
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      const float4 v = good ? *reinterpret_cast<const float4 *>(t + k) : make_float4(nan, nan, nan, nan);
      c[k] = v.x, s[k] = v.y, c[k + 1] = v.z, s[k + 1] = v.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float2 v = good ? t[k] : make_float2(nan, nan);
      c[k] = v.x, s[k] = v.y;
    }
  }
}

// n / d for n < 2^31, d >= 1, by a round-up reciprocal.
struct Divide {
  uint32_t mul, shift;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (__umulhi(mul, n) + n) >> shift; }
};
inline Divide divide_by(uint32_t d) {
  uint32_t shift = 0;
  while ((1ull << shift) < d) ++shift;
  return {(uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1), shift};
}

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

// Launches a kernel that begins with after_earlier_kernels().  It may become resident while the kernel before it on
// the stream is still running (programmatic dependent launch), which hides the 2 us that a launch takes;
// it touches no memory before that kernel has completed.
template <typename... P, typename... A>
int launch(const char *what, void (*kernel)(P...), int64_t blocks, int threads, size_t shared, gar_stream_t stream,
           const A &...args) {
  cudaLaunchAttribute attribute{};
  attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attribute.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3((unsigned)blocks), config.blockDim = dim3((unsigned)threads);
  config.dynamicSmemBytes = shared, config.stream = (cudaStream_t)stream;
  config.attrs = &attribute, config.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&config, kernel, args...);
  return e == cudaSuccess ? GAR_OK : cuda_fail(e, what);
}

// Lets the next such kernel become resident, and waits for the ones before this.
__device__ __forceinline__ void after_earlier_kernels() {
  asm volatile("griddepcontrol.launch_dependents; griddepcontrol.wait;" ::: "memory");
}

inline int refuse(const std::string &why) {
  set_error(why);
  return GAR_EINVAL;
}

// cache.cu
int check_cache(const gar_kv_cache *cache);

}  // namespace gar
