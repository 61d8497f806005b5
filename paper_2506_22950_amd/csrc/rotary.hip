// Rotary positions on rows of Q and K.
//
// Pair j of a head at position p turns by the angle t = p * f_j:
//   out_a = A (x_a cos t - x_b sin t),   out_b = A (x_b cos t + x_a sin t)
// with (a, b) = (j, j + pairs) (halves) or (2j, 2j + 1) (interleaved) and A the
// configuration's amplitude; elements past the rotated part are copied.  The
// gradient of the inputs is the same with -t.
//
// Angles.  p * f_j is formed and reduced in double: at position 2^20 a float
// product is off by 0.06 radian.  With n = round(t * 2/pi) the rest r = t - n pi/2
// (pi/2 in two doubles) lies in [-pi/4, pi/4], where the Taylor sums of sine
// (to r^9) and cosine (to r^10) are within 2e-9 and 2e-10 of them; they are
// evaluated in float, and n mod 4 picks and signs the two.  Sums, products and
// angles stay in 32 bits or more; the one rounding is the output's.
//
// Bound by memory: every row is read and written once, three operations an
// element.  A work-group takes one or more tokens with all their heads, so that
// an angle is computed once per token and layer and read from LDS by every head.
#include "ops.h"

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

// VEC: 16-byte units -- N pairs (32 bytes) of the rotated part, or 16 bytes of the
// rest of a head; else one pair or one element at a time (pairs, strides or
// addresses that 16 bytes do not divide).
template <bool BF, bool INTERLEAVED, bool VEC>
__global__ __launch_bounds__(kRotaryThreads) void rotate_kernel(const RotaryArgs a) {
  using E = Elem<BF>;
  constexpr int N = VEC ? E::N : 1, ES = BF ? 2 : 4;
  __shared__ float2 table[kRotaryTable];
  const int t0 = blockIdx.x * a.tokens_per_wg, nt = min(a.tokens_per_wg, a.tokens - t0);
  const int64_t layer = blockIdx.y;
  for (int i = threadIdx.x; i < nt * a.pairs; i += kRotaryThreads) {
    const int t = t0 + i / a.pairs;
    const int p = a.positions ? a.positions[t] : a.live ? a.pos[t & (kMaxSlots - 1)] : a.first + t;
    float c, s;
    turn_of((double)p * a.freq[i % a.pairs], c, s);
    table[i] = float2{c * a.amplitude, s * a.amplitude * a.sign};
  }
  __syncthreads();
  const int turned = a.pairs / N, units = turned + (a.head_dim - 2 * a.pairs) / N;
  const int heads = a.q.heads + a.k.heads;
  for (int i = threadIdx.x; i < nt * heads * units; i += kRotaryThreads) {
    const int u = i % units, h = i / units % heads, t = i / units / heads;
    if (a.live && !((a.live >> ((t0 + t) & 63)) & 1)) continue;
    const bool is_k = h >= a.q.heads;
    const RotaryRows& r = is_k ? a.k : a.q;
    const int64_t hh = is_k ? h - a.q.heads : h;
    const char* in = r.in + ((int64_t)(t0 + t) * r.in_row + hh * r.in_head + layer * r.in_layer) * ES;
    char* out = r.out + ((int64_t)(t0 + t) * r.out_row + hh * r.out_head + layer * r.out_layer) * ES;
    if (u >= turned) {  // the rest of the head
      const int e = 2 * a.pairs + (u - turned) * N;
      if constexpr (VEC)
        *(u32x4*)(out + e * ES) = *(const u32x4*)(in + e * ES);
      else
        E::copy(out, e, in, e);
      continue;
    }
    const float2* cs = table + t * a.pairs + u * N;
    if constexpr (VEC) {
      const int e0 = INTERLEAVED ? 2 * u * N : u * N, e1 = INTERLEAVED ? e0 + N : a.pairs + u * N;
      const u32x4 x = *(const u32x4*)(in + e0 * ES), y = *(const u32x4*)(in + e1 * ES);
      float lo[N], hi[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (INTERLEAVED) {
          const float p = E::get(2 * j < N ? x : y, 2 * j % N), q = E::get(2 * j < N ? x : y, 2 * j % N + 1);
          const float ra = fmaf(p, cs[j].x, -(q * cs[j].y)), rb = fmaf(q, cs[j].x, p * cs[j].y);
          (2 * j < N ? lo : hi)[2 * j % N] = ra;
          (2 * j < N ? lo : hi)[2 * j % N + 1] = rb;
        } else {
          const float p = E::get(x, j), q = E::get(y, j);
          lo[j] = fmaf(p, cs[j].x, -(q * cs[j].y));
          hi[j] = fmaf(q, cs[j].x, p * cs[j].y);
        }
      }
      *(u32x4*)(out + e0 * ES) = E::pack(lo);
      *(u32x4*)(out + e1 * ES) = E::pack(hi);
    } else {
      const int e0 = INTERLEAVED ? 2 * u : u, e1 = INTERLEAVED ? 2 * u + 1 : a.pairs + u;
      const float p = E::load(in, e0), q = E::load(in, e1);
      E::store(out, e0, fmaf(p, cs[0].x, -(q * cs[0].y)));
      E::store(out, e1, fmaf(q, cs[0].x, p * cs[0].y));
    }
  }
}

// Whether 16-byte units fit rows r.
bool vector_rows(const RotaryRows& r, int n) {
  if (r.heads == 0) return true;
  const int64_t s = r.in_row | r.in_head | r.in_layer | r.out_row | r.out_head | r.out_layer;
  return s % n == 0 && (((uintptr_t)r.in | (uintptr_t)r.out) & 15) == 0;
}

}  // namespace

hipError_t launch_rotate(RotaryArgs& a, bool bf16, bool interleaved, int layers, hipStream_t stream) {
  if (a.tokens == 0 || layers == 0 || a.q.heads + a.k.heads == 0) return hipSuccess;
  const int n = bf16 ? 8 : 4;
  const bool vec = a.pairs % n == 0 && (a.head_dim - 2 * a.pairs) % n == 0 && vector_rows(a.q, n) && vector_rows(a.k, n);
  a.tokens_per_wg = 1;
  const dim3 grid((unsigned)((a.tokens + a.tokens_per_wg - 1) / a.tokens_per_wg), (unsigned)layers);
  void (*const kernels[2][2][2])(const RotaryArgs) = {
      {{rotate_kernel<false, false, false>, rotate_kernel<false, false, true>},
       {rotate_kernel<false, true, false>, rotate_kernel<false, true, true>}},
      {{rotate_kernel<true, false, false>, rotate_kernel<true, false, true>},
       {rotate_kernel<true, true, false>, rotate_kernel<true, true, true>}}};
  hipLaunchKernelGGL(kernels[bf16][interleaved][vec], grid, dim3(kRotaryThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace infs
