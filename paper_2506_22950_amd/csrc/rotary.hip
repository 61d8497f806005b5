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
// an angle is computed once per token and layer and read from LDS by every head;
// it has as many threads as its tokens have units of work, whose first rows are loaded
// while the angles are computed.
#include "ops.h"

#include <algorithm>

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

// What a unit of work is.
enum Unit {
  kElement,  // a pair, or an element behind the rotated part: any sizes and alignment
  kChunk,    // 16 bytes of a head of whole, aligned chunks; halves: its partners, in other chunks, come
             // through LDS
  kPairs     // halves: 16 bytes of first and 16 bytes of second elements (a chunk behind the rotated part),
             // where the pairs too are whole chunks
};

// n / d by inv = ceil(2^32 / d): exact where n d < 2^32 (a work-group has fewer than 2^21 units, at most
// 2^8 to a head, of at most 2^13 heads of one token or 2^8 of several; d = 1 has no inv).
__device__ __forceinline__ int divide(int n, int d, uint32_t inv) { return d == 1 ? n : (int)__umulhi((uint32_t)n, inv); }

template <bool BF>
struct Row {  // one unit of one head
  const char* in;
  char* out;
  int u, t;  // unit of the head, token of the work-group
  bool there;
};

// Unit i of the work-group's nt tokens.
template <bool BF>
__device__ __forceinline__ Row<BF> find_unit(const RotaryArgs& a, int i, int t0, int nt, int units, int64_t layer) {
  constexpr int ES = BF ? 2 : 4;
  Row<BF> r;
  const int heads = a.q.heads + a.k.heads;
  const int head = divide(i, units, a.per_unit), h = head - heads * divide(head, heads, a.per_head);
  r.u = i - head * units;
  r.t = divide(head, heads, a.per_head);
  r.there = r.t < nt && !(a.live && !((a.live >> ((t0 + r.t) & 63)) & 1));
  const bool is_k = h >= a.q.heads;
  const RotaryRows& rows = is_k ? a.k : a.q;
  const int64_t hh = is_k ? h - a.q.heads : h, t = t0 + r.t;
  r.in = rows.in + (t * rows.in_row + hh * rows.in_head + layer * rows.in_layer) * ES;
  r.out = rows.out + (t * rows.out_row + hh * rows.out_head + layer * rows.out_layer) * ES;
  return r;
}

template <bool BF, bool INTERLEAVED, int UNIT>
__global__ __launch_bounds__(INTERLEAVED ? 2 * kRotaryThreads : kRotaryThreads) void rotate_kernel(const RotaryArgs a) {
  using E = Elem<BF>;
  constexpr int N = UNIT == kElement ? 1 : E::N, ES = BF ? 2 : 4;
  // (cos, sin); kChunk: up to N whole columns a token
  __shared__ float2 table[UNIT == kChunk ? kRotaryTable * N : kRotaryTable];
  __shared__ __attribute__((aligned(16))) char chunks[UNIT == kChunk && !INTERLEAVED ? kRotaryThreads * 16 : 16];
  const int t0 = blockIdx.x * a.tokens_per_wg, nt = min(a.tokens_per_wg, a.tokens - t0);
  const int64_t layer = blockIdx.y;
  const int turned = a.pairs / N;  // kPairs, kElement: units of pairs, then of the rest
  const int units = UNIT == kChunk ? a.head_dim / N : turned + (a.head_dim - 2 * a.pairs) / N;
  const int threads = (int)blockDim.x;
  // kChunk: a head's chunks are in one wavefront, so that each holds whole heads (and idle lanes)
  const int lane = threadIdx.x & 63, wave_units = UNIT == kChunk ? 64 / units * units : 64;
  const int step = threads / 64 * wave_units;
  int i = (int)(threadIdx.x >> 6) * wave_units + lane;
  const int total = nt * (a.q.heads + a.k.heads) * units;
  const bool works = lane < wave_units;
  Row<BF> r = find_unit<BF>(a, i, t0, nt, units, layer);
  r.there = r.there && works && i < total;
  // byte offsets of the unit's two halves
  const auto first_of = [&](int u) {
    return (UNIT == kChunk || u < turned ? u * N : 2 * a.pairs + (u - turned) * N) * ES;
  };
  const auto second_of = [&](int u) { return (a.pairs + u * N) * ES; };
  const auto load = [&](const Row<BF>& r, u32x4& x, u32x4& y) {
    if (UNIT == kElement || !r.there) return;
    x = *(const u32x4*)(r.in + first_of(r.u));
    if (UNIT == kPairs && r.u < turned) y = *(const u32x4*)(r.in + second_of(r.u));
  };
  // kChunk: the angles of a chunk are apart in the table, so that those of lanes next to each other lie
  // together (16 lanes read one bank otherwise)
  constexpr int kApart = UNIT != kChunk ? 1 : INTERLEAVED ? N / 2 : N;
  const int columns = (a.pairs + kApart - 1) / kApart;
  const auto place_of = [&](int t, int f) { return (t * kApart + f % kApart) * columns + f / kApart; };
  u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
  load(r, x, y);
  for (int j = threadIdx.x; j < nt * a.pairs; j += threads) {
    const int t = t0 + j / a.pairs;
    const int p = a.positions ? a.positions[t] : a.live ? a.pos[t & (kMaxSlots - 1)] : a.first + t;
    float c, s;
    turn_of((double)p * a.freq[j % a.pairs], c, s);
    table[place_of(j / a.pairs, j % a.pairs)] = float2{c * a.amplitude, s * a.amplitude * a.sign};
  }
  __syncthreads();
  while (true) {
    const float2* cs = table + place_of(r.t, 0);
    if constexpr (UNIT == kElement) {
      if (r.there && r.u >= turned) {
        const int e = 2 * a.pairs + r.u - turned;
        E::copy(r.out, e, r.in, e);
      } else if (r.there) {
        const int e0 = INTERLEAVED ? 2 * r.u : r.u, e1 = INTERLEAVED ? e0 + 1 : a.pairs + e0;
        const float p = E::load(r.in, e0), q = E::load(r.in, e1);
        E::store(r.out, e0, fmaf(p, cs[r.u].x, -(q * cs[r.u].y)));
        E::store(r.out, e1, fmaf(q, cs[r.u].x, p * cs[r.u].y));
      }
    } else if constexpr (UNIT == kPairs) {
      if (r.there && r.u >= turned) {
        __builtin_nontemporal_store(x, (u32x4*)(r.out + first_of(r.u)));
      } else if (r.there) {
        cs += r.u * N;
        float lo[N], hi[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float p = E::get(x, j), q = E::get(y, j);
          lo[j] = fmaf(p, cs[j].x, -(q * cs[j].y));
          hi[j] = fmaf(q, cs[j].x, p * cs[j].y);
        }
        // Past the L2: what a launch leaves there is written back at its end.  Rows that a projection has
        // just written are loaded through the caches: 7424 tokens 25.4 us so, 27.9 us past them (rows from
        // memory: 30.3 and 28.8); both through the caches 30.6 us.
        __builtin_nontemporal_store(E::pack(lo), (u32x4*)(r.out + first_of(r.u)));
        __builtin_nontemporal_store(E::pack(hi), (u32x4*)(r.out + second_of(r.u)));
      }
    } else {
      const char* head = chunks + (threadIdx.x - r.u) * 16;  // the head's elements
      if constexpr (!INTERLEAVED) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last unit's reads are done
        *(u32x4*)(chunks + threadIdx.x * 16) = x;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      if (r.there) {
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int e = r.u * N + j;
          const bool rest = e >= 2 * a.pairs, second = INTERLEAVED ? j & 1 : e >= a.pairs;
          const float own = E::get(x, j);
          float other;
          if constexpr (INTERLEAVED)
            other = E::get(x, j ^ 1);
          else
            other = E::load(head, rest ? e : second ? e - a.pairs : e + a.pairs);
          const float2 w = cs[rest ? 0 : place_of(0, INTERLEAVED ? e >> 1 : second ? e - a.pairs : e)];
          v[j] = rest ? own : fmaf(own, w.x, second ? other * w.y : -(other * w.y));
        }
        __builtin_nontemporal_store(E::pack(v), (u32x4*)(r.out + first_of(r.u)));
      }
    }
    i += step;
    if (i - lane >= total) break;  // the same for all lanes of a wavefront
    r = find_unit<BF>(a, i, t0, nt, units, layer);
    r.there = r.there && works && i < total;
    load(r, x, y);
  }
}

// Whether rows r are aligned to 16 bytes.
bool vector_rows(const RotaryRows& r, int n) {
  if (r.heads == 0) return true;
  const int64_t s = r.in_row | r.in_head | r.in_layer | r.out_row | r.out_head | r.out_layer;
  return s % n == 0 && (((uintptr_t)r.in | (uintptr_t)r.out) & 15) == 0;
}

}  // namespace

hipError_t launch_rotate(RotaryArgs& a, bool bf16, bool interleaved, int layers, hipStream_t stream) {
  if (a.tokens == 0 || layers == 0 || a.q.heads + a.k.heads == 0) return hipSuccess;
  const int n = bf16 ? 8 : 4;
  const bool chunks = a.head_dim % n == 0 && vector_rows(a.q, n) && vector_rows(a.k, n);
  const int unit = !chunks ? kElement : !interleaved && a.pairs % n == 0 ? kPairs : kChunk;
  const int units = unit == kElement ? a.head_dim - a.pairs : unit == kChunk ? a.head_dim / n : (a.head_dim - a.pairs) / n;
  // Tokens of a work-group: one where it fills a work-group's threads, else as many as do, within the
  // table of angles.
  const int64_t per_token = (int64_t)(a.q.heads + a.k.heads) * units;
  a.tokens_per_wg = (int)std::max<int64_t>(1, std::min<int64_t>({kRotaryTable / a.pairs, kRotaryThreads / per_token, a.tokens}));
  const int64_t lanes = unit == kChunk ? per_token * a.tokens_per_wg * 64 / (64 / units * units) : per_token * a.tokens_per_wg;
  // Twice the threads where a compute unit has one work-group at most and a head's units are 16 bytes
  // each (interleaved): 16 tokens of 24 heads of 128 take 3.1 us so, 4.2 us in two turns; 7424 tokens of 40
  // heads 45.7 us so and 37.5 us with 256 threads.
  const int64_t blocks = (a.tokens + a.tokens_per_wg - 1) / a.tokens_per_wg * (int64_t)layers;
  const int most = interleaved && blocks <= kRotaryFewBlocks ? 2 * kRotaryThreads : kRotaryThreads;
  const int threads = (int)std::min<int64_t>(most, (lanes + 63) / 64 * 64);
  a.per_unit = (uint32_t)(((uint64_t(1) << 32) + units - 1) / units);
  const int heads = a.q.heads + a.k.heads;
  a.per_head = (uint32_t)(((uint64_t(1) << 32) + heads - 1) / heads);
#define INFS_ROTATE(bf, il) \
  { rotate_kernel<bf, il, kElement>, rotate_kernel<bf, il, kChunk>, il ? nullptr : rotate_kernel<bf, false, kPairs> }
  void (*const kernels[2][2][3])(const RotaryArgs) = {{INFS_ROTATE(false, false), INFS_ROTATE(false, true)},
                                                      {INFS_ROTATE(true, false), INFS_ROTATE(true, true)}};
#undef INFS_ROTATE
  const int64_t per_launch = kMostBlocks / 2 * a.tokens_per_wg;  // tokens of a launch
  for (int64_t left = a.tokens;; left -= per_launch) {
    a.tokens = (int32_t)std::min(per_launch, left);
    const dim3 grid((unsigned)((a.tokens + a.tokens_per_wg - 1) / a.tokens_per_wg), (unsigned)layers);
    hipLaunchKernelGGL(kernels[bf16][interleaved][unit], grid, dim3(threads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || left <= per_launch) return e;
    for (RotaryRows* r : {&a.q, &a.k}) {
      r->in += per_launch * r->in_row * (bf16 ? 2 : 4);
      r->out += per_launch * r->out_row * (bf16 ? 2 : 4);
    }
    if (a.positions) a.positions += per_launch;
    a.first += (int32_t)per_launch;
  }
}

}  // namespace infs
