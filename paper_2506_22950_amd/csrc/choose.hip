// The choice of the next tokens: from a row z of n logits, its maximum m, the weights w_j = exp((z_j - m) / T).
//
// What is kept is the beginning of the ranking by (z, index), so it is given by one value z* and how many of the
// entries equal to it, by index, are in: top-k fixes them by a count, top-p by a sum, min-p by a value.  The
// token is the first kept entry at which the running sum by index is above u times the whole.
//
// Weights and sums.  Which token it is hangs on where u falls between sums of up to 2^24 terms, so each weight
// is formed in double and held as a whole number of units of 2^-s (s = 62 - log2 n, at most 50): sums are exact,
// the same whatever the order.  A weight below half a unit is none
// (but for u = 0, which takes the first entry of all).  exp2(y) = 2^i exp(f ln 2), |f| <= 1/2, with
// the Taylor sum to f^10 (relative error below 3e-13).
//
// Finding z*.  The entries of a range of values are counted and weighed in kBins bins of equal width; the bin that
// holds the wanted count or sum becomes the range, until its entries are equal.
#include "ops.h"
#include "rows.h"

#include <algorithm>

namespace infs {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 1024, kWavesOf = kThreads / 64, kBins = 2048;

// exp2(y) 2^s, y <= 0, as a whole number.
__device__ __forceinline__ u64 weight(double y, int s) {
  // (bounded first: y is a product, and of a fused product with n only its rounding would be left far down)
  y = fmax(y, -200.0);
  const double n = rint(y), f = (y - n) * 0.69314718055994530942;
  double p = 1.0 / 3628800.0;
  p = fma(p, f, 1.0 / 362880.0);
  p = fma(p, f, 1.0 / 40320.0);
  p = fma(p, f, 1.0 / 5040.0);
  p = fma(p, f, 1.0 / 720.0);
  p = fma(p, f, 1.0 / 120.0);
  p = fma(p, f, 1.0 / 24.0);
  p = fma(p, f, 1.0 / 6.0);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  // below 2^52: the sum's low bits are the number, rounded to nearest
  const double x = ldexp(p, (int)n + s) + 0x1p52;
  return (u64)__double_as_longlong(x) & ((1ull << 52) - 1);
}

__device__ __forceinline__ u64 wave_sum(u64 x) {
  for (int i = 1; i < 64; i <<= 1) x += __shfl_xor(x, i);
  return x;
}

// A row of logits, in vectors of 16 aligned bytes; entries outside it are -inf.
template <bool BF>
struct RowOf {
  using E = Elem<BF>;
  static constexpr int N = E::N, ES = BF ? 2 : 4;
  const char* base;  // of the row's first entry
  int n, off, vectors;
  __device__ __forceinline__ RowOf(const char* p, int n) : base(p), n(n) {
    off = (int)((uintptr_t)p & 15) / ES;
    vectors = (n + off + N - 1) / N;
  }
  __device__ __forceinline__ int index(int v, int j) const { return v * N + j - off; }
  __device__ __forceinline__ void load(int v, float (&x)[N]) const {
    const int i0 = index(v, 0);
    if (i0 >= 0 && i0 + N <= n) {
      const u32x4 w = *(const u32x4*)(base + (int64_t)i0 * ES);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = E::get(w, j) + 0.f;  // -0 counts as 0
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = i0 + j >= 0 && i0 + j < n ? E::load(base, i0 + j) + 0.f : -INFINITY;
    }
  }
};

struct Shared {
  int count[kBins];
  u64 mass[kBins];
  u64 sums[kWavesOf];
  float lows[kWavesOf], highs[kWavesOf];
  int counts[kWavesOf];
  u64 found_mass;
  int found, found_count, flag;
};

template <bool BF>
struct Chooser {
  using R = RowOf<BF>;
  static constexpr int N = R::N;
  R row;
  Shared& sh;
  double c, top;  // log2(e) / T, m
  int s;
  int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  __device__ __forceinline__ u64 w(float z) const { return weight(((double)z - top) * c, s); }

  // The smallest and largest finite value with use(z, index).
  template <class F>
  __device__ __forceinline__ void range(F use, float& lo, float& hi) {
    float a = INFINITY, b = -INFINITY;
    for (int v = threadIdx.x; v < row.vectors; v += kThreads) {
      float x[N];
      row.load(v, x);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (use(x[j])) a = fminf(a, x[j]), b = fmaxf(b, x[j]);
    }
    for (int i = 1; i < 64; i <<= 1) a = fminf(a, __shfl_xor(a, i)), b = fmaxf(b, __shfl_xor(b, i));
    if (lane == 0) sh.lows[wave] = a, sh.highs[wave] = b;
    __syncthreads();
    lo = sh.lows[0], hi = sh.highs[0];
    for (int i = 1; i < kWavesOf; ++i) lo = fminf(lo, sh.lows[i]), hi = fmaxf(hi, sh.highs[i]);
    __syncthreads();
  }

  // z*: in [lo, hi], the value at which the entries above it number `above` < count (weigh `over` < mass, where
  // BY_MASS) and with those equal to it at least that; they are `equal`.
  struct Found {
    float z;
    int above, equal;
    u64 over;
  };
  template <bool BY_MASS>
  __device__ __forceinline__ Found select(float lo, float hi, int count, u64 mass) {
    Found f{hi, 0, 0, 0};
    while (true) {
      // halves, so that the widest range is finite; tiny values scaled up, so that differences are no denormals
      const float up = fmaxf(fabsf(hi), fabsf(lo)) < 0x1p-60f ? 0x1p80f : 0.5f;
      const float width = hi * up - lo * up, by = width > 0.f ? (kBins - 1) / width : 0.f;
      const float hi_up = hi * up;
      const auto bin_of = [&](float z) { return min(kBins - 1, (int)((hi_up - z * up) * by)); };
      for (int i = threadIdx.x; i < kBins; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
      __syncthreads();
      for (int v = threadIdx.x; v < row.vectors; v += kThreads) {
        float x[N];
        row.load(v, x);
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (x[j] >= lo && x[j] <= hi) {
            const int b = bin_of(x[j]);
            atomicAdd(&sh.count[b], 1);
            if (BY_MASS) atomicAdd(&sh.mass[b], w(x[j]));
          }
      }
      __syncthreads();
      // the first bin with which the wanted is reached, by the first wavefront
      if (wave == 0) {
        constexpr int P = kBins / 64;
        int n = 0;
        u64 m = 0;
        for (int i = 0; i < P; ++i) n += sh.count[lane * P + i], m += sh.mass[lane * P + i];
        int before = n;
        u64 under = m;
        for (int i = 1; i < 64; i <<= 1) {
          const int a = __shfl_up(before, i);
          const u64 b = __shfl_up(under, i);
          if (lane >= i) before += a, under += b;
        }
        before += f.above - n, under += f.over - m;  // ahead of the lane's bins
        const bool here = BY_MASS ? under + m >= mass : before + n >= count;
        const u64 mask = __ballot(here);
        const int at = mask ? __builtin_ctzll(mask) : 63;
        if (lane == at) {
          int i = 0;
          for (; i < P - 1; ++i) {
            const int a = sh.count[lane * P + i];
            const u64 b = sh.mass[lane * P + i];
            if (BY_MASS ? under + b >= mass : before + a >= count) break;
            before += a, under += b;
          }
          sh.found = lane * P + i, sh.found_count = before, sh.found_mass = under;
          sh.flag = sh.count[lane * P + i];
        }
      }
      __syncthreads();
      const int bin = sh.found;
      f.above = sh.found_count, f.over = sh.found_mass, f.equal = sh.flag;
      __syncthreads();
      float a, b;
      const float hi0 = hi, lo0 = lo;
      range([&](float z) { return z >= lo0 && z <= hi0 && bin_of(z) == bin; }, a, b);
      if (a >= b || (a == lo0 && b == hi0)) {  // equal (bins of a range of several values always part its ends)
        f.z = b;
        return f;
      }
      lo = a, hi = b;
    }
  }

  // The first index at which the sum of value(z, index) is above target (at least one is).
  template <class F>
  __device__ __forceinline__ int locate(F value, u64 target) {
    int from = 0, to = row.vectors;
    while (true) {
      const int part = ((to - from + kWavesOf - 1) / kWavesOf + 63) / 64 * 64;
      const int a = from + wave * part, b = min(to, a + part);
      u64 sum = 0;
      for (int v = a + lane; v < b; v += 64) {
        float x[N];
        row.load(v, x);
#pragma unroll
        for (int j = 0; j < N; ++j) sum += value(x[j], row.index(v, j));
      }
      sum = wave_sum(sum);
      if (lane == 0) sh.sums[wave] = sum;
      __syncthreads();
      int at = 0;
      u64 under = 0;
      while (at < kWavesOf - 1 && under + sh.sums[at] <= target) under += sh.sums[at++];
      __syncthreads();
      target -= under;
      from += at * part;
      to = min(to, from + part);
      if (part <= 64) break;
    }
    // 64 vectors: by the first wavefront
    if (wave == 0) {
      float x[N];
      const int v = from + lane;
      if (v < to) row.load(v, x);
      u64 sum = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) sum += v < to ? value(x[j], row.index(v, j)) : 0;
      u64 under = sum;
      for (int i = 1; i < 64; i <<= 1) {
        const u64 y = __shfl_up(under, i);
        if (lane >= i) under += y;
      }
      const u64 mask = __ballot(under > target);
      if (lane == (mask ? __builtin_ctzll(mask) : 63)) {
        under -= sum;
        int at = 0;
        bool done = false;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          under += v < to ? value(x[j], row.index(v, j)) : 0;
          if (!done && under > target) at = row.index(v, j), done = true;
        }
        sh.found = at;
      }
    }
    __syncthreads();
    const int at = sh.found;
    __syncthreads();
    return at;
  }

  // Sum of the weights, and number, of the entries with use(z, index).
  template <class F>
  __device__ __forceinline__ u64 total(F use, int& count) {
    u64 sum = 0;
    int n = 0;
    for (int v = threadIdx.x; v < row.vectors; v += kThreads) {
      float x[N];
      row.load(v, x);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (use(x[j], row.index(v, j))) sum += w(x[j]), ++n;
    }
    sum = wave_sum(sum);
    for (int i = 1; i < 64; i <<= 1) n += __shfl_xor(n, i);
    if (lane == 0) sh.sums[wave] = sum, sh.counts[wave] = n;
    __syncthreads();
    sum = 0, n = 0;
    for (int i = 0; i < kWavesOf; ++i) sum += sh.sums[i], n += sh.counts[i];
    __syncthreads();
    count = n;
    return sum;
  }
};

__device__ __forceinline__ bool allowed(const Sampling& p) {
  const double t = p.temperature;
  return (t == 0.0 || (t >= 0x1p-20 && t <= 0x1p20)) && p.top_p >= 0.0 && p.top_p <= 1.0 && p.min_p >= 0.0 &&
         p.min_p <= 1.0 && p.top_k >= 0;
}

template <bool BF>
__global__ __launch_bounds__(kThreads) void choose_kernel(const ChooseArgs a) {
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const Sampling p = a.each ? a.each[r] : a.all;
  const float u = a.uniform[r];
  Chooser<BF> ch{RowOf<BF>((const char*)a.logits + r * a.row_stride * (BF ? 2 : 4), a.vocab), sh, 0.0, 0.0, a.unit};
  constexpr int N = RowOf<BF>::N;
  // the largest and smallest finite values, how many are not masked, and whether any is NaN or +inf
  float lo = INFINITY, hi = -INFINITY;
  int live = 0;
  bool odd = false;
  for (int v = threadIdx.x; v < ch.row.vectors; v += kThreads) {
    float x[N];
    ch.row.load(v, x);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      odd |= !(x[j] < INFINITY);
      if (x[j] > -INFINITY) lo = fminf(lo, x[j]), hi = fmaxf(hi, x[j]), ++live;
    }
  }
  for (int i = 1; i < 64; i <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, i)), hi = fmaxf(hi, __shfl_xor(hi, i));
    live += __shfl_xor(live, i);
  }
  if (ch.lane == 0) sh.lows[ch.wave] = lo, sh.highs[ch.wave] = hi, sh.counts[ch.wave] = live;
  odd = __syncthreads_or(odd);
  live = 0;
  for (int i = 0; i < kWavesOf; ++i) lo = fminf(lo, sh.lows[i]), hi = fmaxf(hi, sh.highs[i]), live += sh.counts[i];
  __syncthreads();
  if (odd || live == 0 || !(u >= 0.f && u < 1.f) || !allowed(p)) {
    if (threadIdx.x == 0) {
      a.token[r] = -1;
      if (a.logprob) a.logprob[r] = NAN;
      if (a.kept) a.kept[r] = 0;
    }
    return;
  }
  ch.c = 1.4426950408889634074 / (p.temperature == 0.0 ? 1.0 : p.temperature);
  ch.top = hi;
  const u64 one = 1ull << a.unit;
  // kept: above z*, and of those equal to it the first `equal` of `ties`
  float z = lo;
  int ties = 0, equal = 0;
  const bool by_count = p.top_k > 0 && p.top_k < live, by_mass = p.top_p > 0.0 && p.top_p < 1.0;
  u64 limit = ~0ull;  // what the entries kept by count weigh
  if (by_count) {
    const auto f = ch.template select<false>(lo, hi, p.top_k, 0);
    z = f.z, ties = f.equal, equal = p.top_k - f.above;
  }
  if (by_mass) {
    int n;
    const float z0 = z;
    limit = ch.total([&](float x, int) { return by_count ? x > z0 : x > -INFINITY; }, n) + (by_count ? equal * ch.w(z0) : 0);
    // entries whose predecessors weigh less than the share: up to the first whose sum with them reaches it
    const u64 share = (u64)ceil(p.top_p * (double)limit);
    const auto f = ch.template select<true>(z0, hi, 0, share);
    const u64 each = ch.w(f.z);
    const int most = by_count && f.z == z0 ? equal : f.equal;
    u64 k = each ? (share - f.over + each - 1) / each : most;
    z = f.z, ties = f.equal, equal = k < (u64)most ? (int)k : most;
  }
  int last = INT32_MAX;  // index of the last kept entry that equals z*
  if ((by_count || by_mass) && equal < ties)
    last = ch.locate([&](float x, int) -> u64 { return x == z ? 1 : 0; }, (u64)(equal - 1));
  const bool ranked = by_count || by_mass;
  const double least = p.min_p;
  const auto kept = [&](float x, int i) {
    if (!(x > -INFINITY)) return false;
    if (ranked && !(x > z || (x == z && i <= last))) return false;
    return !(least > 0.0) || x == hi || (double)ch.w(x) >= least * (double)one;
  };
  int n;
  const u64 sum = ch.total(kept, n);
  const u64 target = (u64)((double)u * (double)sum);
  // u = 0 takes the first entry of any weight at all (in double), however small the unit makes it
  const int token = u == 0.f
                        ? ch.locate([&](float x, int i) -> u64 { return kept(x, i) && ((double)x - ch.top) * ch.c > -1074.0; }, 0)
                        : ch.locate([&](float x, int i) -> u64 { return kept(x, i) ? ch.w(x) : 0; },
                                    target < sum ? target : sum - 1);
  if (threadIdx.x == 0) {
    a.token[r] = token;
    if (a.logprob) {
      const double y = ((double)Elem<BF>::load(ch.row.base, token) - ch.top) * ch.c;
      a.logprob[r] = (float)((y + a.unit) * 0.69314718055994530942 - log((double)sum));
    }
    if (a.kept) a.kept[r] = n;
  }
}

}  // namespace

hipError_t launch_choose(ChooseArgs& a, bool bf16, hipStream_t stream) {
  a.unit = 62;
  while ((int64_t(1) << (62 - a.unit)) < a.vocab) --a.unit;
  a.unit = std::min(a.unit, 50);
  if (bf16)
    hipLaunchKernelGGL(choose_kernel<true>, dim3(a.rows), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(choose_kernel<false>, dim3(a.rows), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace infs
