// What the kernels on rows of heads share (rotary.hip, norm.hip): elements of a
// type, sine and cosine of an angle, division by a host constant.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace infs {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

__device__ __forceinline__ void turn_of(double t, float& c, float& s) {
  const double n = rint(t * 0.63661977236758134308);  // 2 / pi
  double r = fma(-n, 1.57079632679489661923, t);      // pi / 2, high part
  r = fma(-n, 6.123233995736766e-17, r);              // and the rest of it
  const float x = (float)r, z = x * x;
  const float sx =
      x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float cx = fmaf(
      z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int q = (int)((long long)n & 3);
  const float a = (q & 1) ? cx : sx, b = (q & 1) ? sx : cx;
  s = (q & 2) ? -a : a;
  c = ((q + 1) & 2) ? -b : b;
}

template <bool BF>
struct Elem;
template <>
struct Elem<true> {
  static constexpr int N = 8;  // elements of 16 bytes
  static __device__ __forceinline__ float get(const u32x4& v, int i) {
    const uint32_t w = v[i >> 1];
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  static __device__ __forceinline__ uint32_t bits(float x) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = bits(x[2 * i]) | (bits(x[2 * i + 1]) << 16);
    return r;
  }
  static __device__ __forceinline__ float load(const char* p, int64_t i) {
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
  }
  static __device__ __forceinline__ void store(char* p, int64_t i, float x) { ((uint16_t*)p)[i] = (uint16_t)bits(x); }
  static __device__ __forceinline__ void copy(char* d, int64_t j, const char* p, int64_t i) {
    ((uint16_t*)d)[j] = ((const uint16_t*)p)[i];
  }
};
template <>
struct Elem<false> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const u32x4& v, int i) { return __uint_as_float(v[i]); }
  static __device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
    return r;
  }
  static __device__ __forceinline__ float load(const char* p, int64_t i) { return ((const float*)p)[i]; }
  static __device__ __forceinline__ void store(char* p, int64_t i, float x) { ((float*)p)[i] = x; }
  static __device__ __forceinline__ void copy(char* d, int64_t j, const char* p, int64_t i) {
    ((uint32_t*)d)[j] = ((const uint32_t*)p)[i];
  }
};

// n / d by inv = ceil(2^32 / d): exact where n d < 2^32 (a work-group has fewer than 2^21 units, at most
// 2^8 to a head, of at most 2^13 heads of one token or 2^8 of several; d = 1 has no inv).
__device__ __forceinline__ int divide(int n, int d, uint32_t inv) { return d == 1 ? n : (int)__umulhi((uint32_t)n, inv); }

}  // namespace
}  // namespace infs
