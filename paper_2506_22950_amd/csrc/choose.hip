// The choice of the next tokens: from a row z of n logits, its maximum m, the weights w_j = exp((z_j - m) / T).
//
// What is kept is the beginning of the ranking by (z, index), so it is given by one value z* and how many of the
// entries equal to it, by index, are in: top-k fixes them by a count, top-p by a sum, min-p by a value.  The
// token is the first kept entry at which the running sum by index is above u times the whole.
//
// Weights and sums.  Which token it is hangs on where u falls between sums of up to 2^24 terms, so each weight
// is formed in double and, where entries are ranked, held as a whole number of units of 2^-s (s = 62 - log2 n, at most
// 50): sums are exact, the same whatever the order.  A weight below half a unit is none (but for u = 0, which takes the
// first entry of all).  The whole distribution is added up in double, in an order that sizes and alignment fix.
//
// Two launches, each over pieces of rows (kPieceThreads threads, at most 32 entries of each in registers); the last
// piece of a row to arrive joins them (nothing waits).
//   weigh   reads the row: its maximum and, as the way of choosing needs, the sum of its weights and a histogram over
//           the logarithm of the weights (kBins bins of 1/kBinsPerOctave octave below the maximum).  Without a
//           filter the join takes the token; else it finds the bin in which z* lies.
//   gather  reads the row again (out of a cache): entries of that bin, and for small top-k those above it too, go
//           into a list, which the join ranks; the weights above it go into sums.  The join cuts the list at z*
//           and finds the token by the sums.
// Pieces weigh by their own maximum; the join scales their sums in double, in piece order.  Where all rows go one way,
// the whole distribution and a small top-k take one launch (whole_kernel, top_kernel).
//
// Rows for which that does not do (a list of more than kList entries, as where logits are equal; z* beyond the bins;
// a large top-k with top-p; u = 0) the last piece takes alone: the entries of a range of values are counted and
// weighed in bins of equal width, and the bin that holds the wanted count or sum becomes the range, until its
// entries are equal.
#include "ops.h"
#include "rows.h"

#include <algorithm>

namespace infs {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = kPieceThreads, kWavesOf = kThreads / 64, kRangeBins = 2048;

// ln of exp2(y)'s share of a sum of weights of unit 2^-s; 0 where it is all of it.
template <class T>
__device__ __forceinline__ double log_share(double y, T sum, int s) {
  return y * 0.69314718055994530942 - log(ldexp((double)sum, -s));
}

// exp2(y) 2^s, y <= 0 (from -200 on).  2^f on [-1/2, 1/2] by the polynomial of degree 8 of the least relative error (by
// exchange), its constant then set to 1, so that equal largest entries weigh 1 (1e-12); n = round(y) by an addition
// that leaves it in the sum's low bits.
__device__ __forceinline__ double power(double y, int s) {
  // (bounded first: y is a product, and of a fused product with n only its rounding would be left far down)
  y = fmax(y, -200.0);
  const double t = y + 0x1.8p52, f = y - (t - 0x1.8p52);
  double p = 1.3175858111453815e-06;
  p = fma(p, f, 1.5309737421943565e-05);
  p = fma(p, f, 0.00015403851748740978);
  p = fma(p, f, 0.0013333452062248836);
  p = fma(p, f, 0.009618128542862378);
  p = fma(p, f, 0.05550410939341711);
  p = fma(p, f, 0.24022650698880368);
  p = fma(p, f, 0.6931471805465141);
  p = fma(p, f, 1.0);
  const int n = (int)(uint32_t)__double_as_longlong(t) + s;
  return __longlong_as_double(__double_as_longlong(p) + ((long long)n << 52));
}

// The same as a whole number: added to 2^52, the sum's low bits are it, rounded to nearest.
__device__ __forceinline__ u64 weight(double y, int s) {
  return (u64)__double_as_longlong(power(y, s) + 0x1p52) & ((1ull << 52) - 1);
}

// x of another lane, by a move between lanes (DPP control C, of the rows in ROWS), 0 where there is none.
template <int C, int ROWS, class T>
__device__ __forceinline__ T moved(T x) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "one or two registers");
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), C, ROWS, 0xf, false));
  } else {
    const long long v = __builtin_bit_cast(long long, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, C, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), C, ROWS, 0xf, false);
    return __builtin_bit_cast(T, (long long)((u64)hi << 32 | lo));
  }
}

// Running sum over a wavefront: shifts by 1, 2, 4, 8 in rows of 16, then rows' last lanes into the rows behind.
template <class T>
__device__ __forceinline__ T wave_running(T x) {
  x += moved<0x111, 0xf>(x);
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);
  x += moved<0x143, 0xc>(x);
  return x;
}

// The value of lane 63, the same in all.
template <class T>
__device__ __forceinline__ T last_lane(T x) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
  } else {
    const long long v = __builtin_bit_cast(long long, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)v, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 63);
    return __builtin_bit_cast(T, (long long)((u64)hi << 32 | lo));
  }
}

template <class T>
__device__ __forceinline__ T wave_sum(T x) {
  return last_lane(wave_running(x));
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
  // As it lies in memory, -inf outside the row.
  __device__ __forceinline__ u32x4 packed(int v) const {
    const int i0 = index(v, 0);
    if (i0 >= 0 && i0 + N <= n) return *(const u32x4*)(base + (int64_t)i0 * ES);
    float x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = i0 + j >= 0 && i0 + j < n ? E::load(base, i0 + j) : -INFINITY;
    return E::pack(x);
  }
  __device__ __forceinline__ float at(int i) const { return E::load(base, i) + 0.f; }  // -0 counts as 0
};

struct Shared {
  int count[kRangeBins];
  u64 mass[kRangeBins];
  u64 sums[kWavesOf];
  float lows[kWavesOf], highs[kWavesOf];
  int counts[kWavesOf];
  u64 found_mass;
  int found, found_count, flag;
};

template <bool BF>
struct Chooser {
  using R = RowOf<BF>;
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
#pragma unroll 1
    for (int i = threadIdx.x; i < row.n; i += kThreads) {
      const float x = row.at(i);
      if (use(x)) a = fminf(a, x), b = fmaxf(b, x);
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
      const float width = hi * up - lo * up, by = width > 0.f ? (kRangeBins - 1) / width : 0.f;
      const float hi_up = hi * up;
      const auto bin_of = [&](float z) { return min(kRangeBins - 1, (int)((hi_up - z * up) * by)); };
      for (int i = threadIdx.x; i < kRangeBins; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
      __syncthreads();
#pragma unroll 1
      for (int i = threadIdx.x; i < row.n; i += kThreads) {
        const float x = row.at(i);
        if (x >= lo && x <= hi) {
          const int b = bin_of(x);
          atomicAdd(&sh.count[b], 1);
          if (BY_MASS) atomicAdd(&sh.mass[b], w(x));
        }
      }
      __syncthreads();
      // the first bin with which the wanted is reached, by the first wavefront
      if (wave == 0) {
        constexpr int P = kRangeBins / 64;
        int n = 0;
        u64 m = 0;
        #pragma unroll 1
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
    int from = 0, to = row.n;
    while (true) {
      const int part = ((to - from + kWavesOf - 1) / kWavesOf + 63) / 64 * 64;
      const int a = from + wave * part, b = min(to, a + part);
      u64 sum = 0;
#pragma unroll 1
      for (int i = a + lane; i < b; i += 64) sum += value(row.at(i), i);
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
    // 64 entries: by the first wavefront
    if (wave == 0) {
      const int i = from + lane;
      const u64 under = wave_running(i < to ? value(row.at(i), i) : 0);
      const u64 mask = __ballot(under > target);
      if (lane == 0) sh.found = from + (mask ? __builtin_ctzll(mask) : 0);
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
#pragma unroll 1
    for (int i = threadIdx.x; i < row.n; i += kThreads) {
      const float x = row.at(i);
      if (use(x, i)) sum += w(x), ++n;
    }
    sum = wave_sum(sum), n = wave_sum(n);
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
         p.min_p <= 1.0 && p.top_k >= 0 && p.reserved == 0;
}

// A whole row by one work-group.  (Its loops are kept rolled: it is inlined into kernels whose registers it should not
// raise, and as a call it took scratch memory, for which a launch pays.)
template <bool BF>
__device__ __forceinline__ void choose_row(const ChooseArgs& a, int64_t r, Shared& sh) {
  __syncthreads();  // what else lay in sh is no longer read
  const Sampling p = a.each ? a.each[r] : a.all;
  const float u = a.uniform[r];
  Chooser<BF> ch{RowOf<BF>((const char*)a.logits + r * a.row_stride * (BF ? 2 : 4), a.vocab), sh, 0.0, 0.0, a.unit};
  // the largest and smallest finite values, how many are not masked, and whether any is NaN or +inf
  float lo = INFINITY, hi = -INFINITY;
  int live = 0;
  bool odd = false;
#pragma unroll 1
  for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
    const float x = ch.row.at(i);
    odd |= !(x < INFINITY);
    if (x > -INFINITY) lo = fminf(lo, x), hi = fmaxf(hi, x), ++live;
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
      a.logprob[r] = (float)(log_share(y, sum, a.unit));
    }
    if (a.kept) a.kept[r] = n;
  }
}


// ---- pieces -------------------------------------------------------------------
constexpr int kPieceWaves = kPieceThreads / 64;

template <class T>
__device__ __forceinline__ void publish(T* p, T x) {  // past the caches of this XCD
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T collect(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Whether this work-group is the last of `pieces` to come here, with what it published.  Leaves the counter 0.
__device__ __forceinline__ bool arrive(int32_t* counter, int pieces) {
  __shared__ bool last;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);  // this thread's stores have reached the coherence point
  __syncthreads();
  if (threadIdx.x == 0) {
    last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pieces - 1;
    if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
  }
  __syncthreads();
  return last;
}

// A running sum over the threads of a work-group, in thread order; x becomes the sum up to and with it.  Returns the
// whole.  scratch: kPieceWaves.
template <class T>
__device__ __forceinline__ T running(T& x, T* scratch) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_running(x);
  __syncthreads();
  if (lane == 63) scratch[wave] = x;
  __syncthreads();
  T whole = 0, ahead = 0;
#pragma unroll
  for (int i = 0; i < kPieceWaves; ++i) {
    if (i == wave) ahead = whole;
    whole += scratch[i];
  }
  x += ahead;
  return whole;
}

// Order of a value as an unsigned number, and back; keys rank by value, then by the lower index.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z);
  return b ^ ((b & 0x80000000u) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o ^ ((o & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ u64 key_of(float z, int i) { return (u64)order_of(z) << 32 | (0xffffffffu - (uint32_t)i); }
__device__ __forceinline__ int index_of(u64 key) { return (int)(0xffffffffu - (uint32_t)key); }

// How a row is chosen from, as its parameters say.
struct Way {
  double c;     // log2(e) / T
  float bins;   // kBinsPerOctave times that: a value's bin is floor(z * bins)
  bool by_count, by_mass, by_share, ok;
  __device__ __forceinline__ Way(const Sampling& p, float u, int vocab) {
    ok = u >= 0.f && u < 1.f && allowed(p);
    c = 1.4426950408889634074 / (p.temperature == 0.0 ? 1.0 : p.temperature);
    bins = (float)(c * kBinsPerOctave);
    by_count = p.top_k > 0 && p.top_k < vocab;
    by_mass = p.top_p > 0.0 && p.top_p < 1.0;
    by_share = p.min_p > 0.0;
  }
  __device__ __forceinline__ bool whole() const { return !by_count && !by_mass && !by_share; }
};

__device__ __forceinline__ void write_token(const ChooseArgs& a, int64_t r, int token, double logprob, int kept) {
  a.token[r] = token;
  if (a.logprob) a.logprob[r] = (float)logprob;
  if (a.kept) a.kept[r] = kept;
}

// The place in a wavefront's 64 vectors at which the running sum of value(z, index) is above target, by a whole
// work-group (each thread an entry or less): the index, left in *found.  first: the first of these vectors.
template <bool BF, class F>
__device__ __forceinline__ void find_entry(const RowOf<BF>& row, int first, u64 target, F value, u64* scratch, int* found) {
  constexpr int N = RowOf<BF>::N;
  static_assert(64 * N <= kPieceThreads, "an entry a thread");
  const int t = threadIdx.x, i = row.index(first, 0) + t;
  u64 w = 0;
  if (t < 64 * N && i >= 0 && i < row.n) w = value(row.at(i), i);
  u64 sum = w;
  running(sum, scratch);
  if (w > 0 && sum > target && sum - w <= target) *found = i;
  __syncthreads();
}

// A piece of a row: vector i of a thread is i * kPieceThreads behind its first.
template <bool BF>
struct Piece {
  static constexpr int N = RowOf<BF>::N, V = kPieceVectors;
  u32x4 x[V];
  RowOf<BF> row;
  int first, batches, wave, lane;
  __device__ __forceinline__ Piece(const ChooseArgs& a, int64_t r, int piece)
      : row((const char*)a.logits + r * a.row_stride * (BF ? 2 : 4), a.vocab) {
    wave = threadIdx.x >> 6, lane = threadIdx.x & 63, batches = a.batches;
    first = piece * batches * kPieceThreads;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < batches) x[i] = row.packed(vector(i));
  }
  __device__ __forceinline__ int vector(int i) const { return first + i * kPieceThreads + (int)threadIdx.x; }
  __device__ __forceinline__ float at(int i, int j) const { return Elem<BF>::get(x[i], j) + 0.f; }  // -0 counts as 0
};

// keys[0 .. n) in descending order, in the first `size` (a power of two, zeros behind n).
__device__ __forceinline__ void sort_keys(u64* keys, int n, int size) {
  if (n <= kPieceThreads) {  // by each key's rank, as many comparisons as keys (28 to 45 steps with barriers otherwise)
    __syncthreads();
    const u64 own = (int)threadIdx.x < n ? keys[threadIdx.x] : 0;
    int rank = 0;
    if ((int)(threadIdx.x & ~63u) < n) {
#pragma unroll 8
      for (int i = 0; i < n; ++i) rank += keys[i] > own;
    }
    __syncthreads();
    if ((int)threadIdx.x < n) keys[rank] = own;
    __syncthreads();
    return;
  }
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < size / 2; i += kPieceThreads) {
        const int x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x + j;
        const u64 s = keys[x], t = keys[y];
        if ((s < t) == ((x & k) == 0)) keys[x] = t, keys[y] = s;
      }
    }
  __syncthreads();
}

// A row's list of n keys into LDS, ranked.
__device__ __forceinline__ void rank_list(u64* keys, const u64* list, int n) {
  int size = 64;
  while (size < n) size <<= 1;
  for (int i = threadIdx.x; i < size; i += kPieceThreads) keys[i] = i < n ? collect(list + i) : 0;
  sort_keys(keys, n, size);
}

// What a ranked list keeps: its first `count` entries.  upto[i]: an entry's weight, 0 if it is not kept; target: u of
// the whole sum.  over, over_count: the sum and number of the entries above the list.
struct Kept {
  int count;
  u64 whole, target;
};
template <class F>
__device__ __forceinline__ Kept cut_list(const Sampling& p, const Way& way, float u, int unit, float m, bool count, double whole,
                                         u64 over, int over_count, const u64* keys, u64* upto, int n, F w_of, u64* scratch,
                                         int* counts) {
  constexpr int P = kList / kPieceThreads;
  const int each = (n + kPieceThreads - 1) / kPieceThreads, first = threadIdx.x * each;  // of a thread
  u64 w[P], own = 0, limited = 0;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    w[k] = 0;
    if (k < each && first + k < n) {
      w[k] = w_of(value_of(keys[first + k]));
      own += w[k];
      if (first + k < p.top_k) limited += w[k];
    }
  }
  u64 under = own;
  running(under, scratch);
  under -= own;
  // the share that an entry's predecessors weigh less than: of all entries, or of a list that has all of the top_k
  u64 share = ~0ull;
  if (way.by_mass) share = (u64)ceil(p.top_p * (count ? (double)running(limited, scratch) : whole));
  const double least = p.min_p * (double)(1ull << unit);
  int kept = 0;
  u64 sum = 0;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int i = first + k;
    if (k < each && i < n) {
      const bool in = (!count || over_count + i < p.top_k) && (!way.by_mass || over + under < share) &&
                      (!way.by_share || value_of(keys[i]) == m || (double)w[k] >= least);
      kept += in;
      under += w[k];
      upto[i] = in ? w[k] : 0;
      sum += upto[i];
    }
  }
  Kept x;
  x.count = running(kept, counts);  // what leaves an entry in leaves those before it in
  x.whole = over + running(sum, scratch);
  x.target = (u64)((double)u * (double)x.whole);
  if (x.target >= x.whole) x.target = x.whole - 1;
  return x;
}

// The entry at which the kept weights by index are above the target, where all of them are in the list; its index in
// *found.
__device__ __forceinline__ void find_listed(const Kept& x, u64* keys, const u64* upto, u64* scratch, int* found) {
  constexpr int P = kList / kPieceThreads;
  // keys by index (the lowest is the highest) with their places in the ranking
  const int m = x.count;
  int size = 64;
  while (size < m) size <<= 1;
  __syncthreads();
  for (int i = threadIdx.x; i < size; i += kPieceThreads) keys[i] = i < m ? (u64)(uint32_t)keys[i] << 32 | (uint32_t)i : 0;
  sort_keys(keys, m, size);
  const int each = (m + kPieceThreads - 1) / kPieceThreads, first = threadIdx.x * each;
  u64 v[P], own = 0;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    v[k] = k < each && first + k < m ? upto[(uint32_t)keys[first + k]] : 0;
    own += v[k];
  }
  u64 ahead = own;
  running(ahead, scratch);
  ahead -= own;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    if (v[k] > 0 && ahead <= x.target && ahead + v[k] > x.target) *found = index_of((u64)(keys[first + k] >> 32));
    ahead += v[k];
  }
  __syncthreads();
}

// The keys of a thread's `here` entries with in(z) go to the list in LDS (what does not fit is counted), a place for all
// of them at once.
template <bool BF, class F>
__device__ __forceinline__ void list_entries(const Piece<BF>& pc, int here, F in, u64* keys, int* listed) {
  if (here == 0) return;
  int at = atomicAdd(listed, here);
#pragma unroll
  for (int i = 0; i < Piece<BF>::V; ++i)
#pragma unroll
    for (int j = 0; j < Piece<BF>::N && i < pc.batches; ++j) {
      const float z = pc.at(i, j);
      if (!in(z)) continue;
      if (at < kList) keys[at] = key_of(z, pc.row.index(pc.vector(i), j));
      ++at;
    }
}

// Weight of an entry `f` of a bin above its beginning, in units of 2^-16 of the least weight in the bin: kPieceThreads *
// kPieceVectors * 8 of them, 2^(1/32) at most each, fit 32 bits.
__device__ __forceinline__ uint32_t bin_mass(float f) {
  return (uint32_t)(__builtin_amdgcn_exp2f(f * (1.f / kBinsPerOctave)) * 65536.f + 0.5f);
}
static_assert(kPieceThreads * kPieceVectors * 8 * 66974ull < (1ull << 32), "a bin's sum");

// The weighing launch.  101 rows of 50257 in fp32, top-p and min-p: 21 us, of which 2.5 until the piece is there, 5 for the
// weights (a degree-8 polynomial in double each) and the bins, 6.5 for the join; the rest is the launch and what CUs with two
// pieces take longer.
template <bool BF>
__global__ __launch_bounds__(kPieceThreads, 4) void weigh_kernel(const ChooseArgs a) {
  constexpr int N = RowOf<BF>::N, V = Piece<BF>::V, W = kPieceWaves;
  __shared__ __attribute__((aligned(16))) char lds[sizeof(Shared)];
  uint32_t* bins = (uint32_t*)lds;
  __shared__ u64 scratch[W];
  __shared__ double dscratch[W];
  __shared__ float tops[W];
  __shared__ int lives[W], found, found_piece;
  __shared__ u64 inner;
  const int rec = blockIdx.x, local = rec / a.pieces, piece = rec - local * a.pieces;
  const int64_t r = a.row0 + local;
  const Sampling p = a.each ? a.each[r] : a.all;
  const float u = a.uniform[r];
  const Way way(p, u, a.vocab);
  RowState& state = a.state[local];
  if (!way.ok) {
    if (piece == 0 && threadIdx.x == 0) state.mode = kDone, write_token(a, r, -1, NAN, 0);
    return;
  }
  Piece<BF> pc(a, r, piece);
  for (int i = threadIdx.x; i < kBins; i += kPieceThreads) bins[i] = 0;
  float m = -INFINITY;
  int live = 0;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < N && i < pc.batches; ++j) {
      const float z = pc.at(i, j);
      odd |= !(z < INFINITY);
      m = fmaxf(m, z);
      live += z > -INFINITY;
    }
  for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i)), live += __shfl_xor(live, i);
  if (pc.lane == 0) tops[pc.wave] = m, lives[pc.wave] = live;
  odd = __syncthreads_or(odd);
  m = tops[0], live = lives[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, tops[i]), live += lives[i];
  const bool weigh = way.whole() || (way.by_mass && !way.by_count);
  const bool binned = way.by_count ? p.top_k <= kListCount || !way.by_mass : way.by_mass;
  const float top_bin = floorf(m * way.bins);
  u64 sum = 0;
  if (m > -INFINITY && !odd && (weigh || binned)) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i >= pc.batches) break;
      u64 part = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float z = pc.at(i, j);
        const u64 w = weigh && z > -INFINITY ? weight(((double)z - m) * way.c, a.unit) : 0;
        part += w;
        if (binned) {
          const float g = z * way.bins, f = floorf(g), b = top_bin - f;
          if (b < (float)kBins) atomicAdd(&bins[(int)b], way.by_count ? 1u : bin_mass(g - f));
        }
      }
      if (weigh) {
        part = wave_sum(part);
        sum += part;
        if (way.whole() && pc.lane == 0) publish(a.subs + ((int64_t)rec * V + i) * W + pc.wave, part);
      }
    }
    if (weigh) {
      __syncthreads();
      if (pc.lane == 0) scratch[pc.wave] = sum;
    }
  } else {
    __syncthreads();
    if (pc.lane == 0) {
      scratch[pc.wave] = 0;
      if (way.whole())
        for (int i = 0; i < pc.batches; ++i) publish(a.subs + ((int64_t)rec * V + i) * W + pc.wave, (u64)0);
    }
  }
  __syncthreads();
  PieceState& mine = a.piece[rec];
  if (threadIdx.x == 0) {
    sum = 0;
    for (int i = 0; i < W; ++i) sum += scratch[i];
    publish(&mine.top, odd ? NAN : m);
    publish(&mine.live, live);
    publish(&mine.sum, weigh ? sum : 0);
  }
  if (binned)
    for (int i = threadIdx.x; i < kBins; i += kPieceThreads) publish(a.bins + (int64_t)rec * kBins + i, bins[i]);
  if (!arrive(a.arrived + local * kCounterStride, a.pieces)) return;

  // ---- the row ----
  const PieceState* all = a.piece + (int64_t)local * a.pieces;
  m = -INFINITY, live = 0, odd = false;
  for (int i = threadIdx.x; i < a.pieces; i += kPieceThreads) {
    const float t = collect(&all[i].top);
    odd |= t != t;
    m = fmaxf(m, t);
    live += collect(&all[i].live);
  }
  for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i)), live += __shfl_xor(live, i);
  if (pc.lane == 0) tops[pc.wave] = m, lives[pc.wave] = live;
  odd = __syncthreads_or(odd);
  m = tops[0], live = lives[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, tops[i]), live += lives[i];
  if (odd || live == 0) {
    if (threadIdx.x == 0) state.mode = kDone, write_token(a, r, -1, NAN, 0);
    return;
  }
  // pieces' sums in units of the row's maximum: thread t has pieces t * per .. (a piece's scale is 2^-unit and more)
  const int per = (a.pieces + kPieceThreads - 1) / kPieceThreads, from_piece = min(a.pieces, (int)threadIdx.x * per),
            to_piece = min(a.pieces, from_piece + per);
  const auto scale_of = [&](float t) { return power(((double)t - m) * way.c, 0); };
  double whole = 0.0, before = 0.0;
  if (weigh) {
    double own = 0.0;
    for (int i = from_piece; i < to_piece; ++i) {
      const u64 w = collect(&all[i].sum);
      if (w) own += (double)w * scale_of(collect(&all[i].top));
    }
    before = own;
    whole = running(before, dscratch);
    before -= own;
  }
  if (way.whole()) {
    if (u == 0.f) {
      if (threadIdx.x == 0) state.mode = kDone;
      choose_row<BF>(a, r, *(Shared*)lds);
      return;
    }
    const double target = (double)u * whole;
    if (threadIdx.x == 0) found = -1, found_piece = -1;
    __syncthreads();
    // running sums of one thread and of the next may differ by a rounding: the first piece wins, and the last piece of
    // any weight takes what is left
    double with = before;
    for (int i = from_piece; i < to_piece; ++i) {
      const u64 w = collect(&all[i].sum);
      if (!w) continue;
      with += (double)w * scale_of(collect(&all[i].top));
      if (with > target) atomicMin((unsigned*)&found_piece, (unsigned)i);
      atomicMax(&found, i);
    }
    __syncthreads();
    const int at = found_piece >= 0 ? found_piece : found;
    if (at >= from_piece && at < to_piece) {
      double under = before;
      for (int i = from_piece; i < at; ++i) {
        const u64 w = collect(&all[i].sum);
        if (w) under += (double)w * scale_of(collect(&all[i].top));
      }
      const u64 w = collect(&all[at].sum);
      const double rest = fmax(0.0, (target - under) / scale_of(collect(&all[at].top)));
      inner = rest < (double)w ? min((u64)rest, w - 1) : w - 1;
    }
    __syncthreads();
    u64 want = inner;
    const float t = collect(&all[at].top);
    // its wavefront's batch
    const u64* subs = a.subs + ((int64_t)local * a.pieces + at) * V * W;
    u64 part = (int)threadIdx.x < a.batches * W ? collect(subs + threadIdx.x) : 0, upto = part;
    running(upto, scratch);
    if (part > 0 && upto > want && upto - part <= want) found = threadIdx.x, inner = upto - part;
    __syncthreads();
    want -= inner;
    const int sub = found;
    __syncthreads();
    const int from = at * a.batches * kPieceThreads + sub / W * kPieceThreads + sub % W * 64;
    find_entry<BF>(pc.row, from, want,
                   [&](float z, int) -> u64 { return z > -INFINITY ? weight(((double)z - t) * way.c, a.unit) : 0; }, scratch,
                   &found);
    if (threadIdx.x == 0) {
      const double y = ((double)Elem<BF>::load(pc.row.base, found) - m) * way.c;
      write_token(a, r, found, log_share(y, whole, a.unit), live);
      state.mode = kDone;
    }
    return;
  }
  // The bins of the entries to list.  hi_bin, lo_bin: floor(z bins) of the highest and lowest.
  const float row_bin = floorf(m * way.bins);
  const bool count = way.by_count && p.top_k < live, mass = way.by_mass;
  int mode = kSums;
  float lo_bin = -INFINITY, hi_bin = -INFINITY;
  // (bins are whole numbers of float32)
  if (!(fabsf(row_bin) < 0x1p22f) || (mass && way.by_count && (p.top_k > kListCount || !count))) mode = kLeft;
  if (mode != kLeft && (count || mass)) {
    const bool by_mass = !count;
    // where the pieces' bin 0 is in the row's (kBins: nowhere)
    int* offs = (int*)lds;
    static_assert(sizeof(lds) >= kChoosePieces * sizeof(int), "bins of the pieces");
    for (int i = threadIdx.x; i < a.pieces; i += kPieceThreads) {
      const float off = row_bin - floorf(collect(&all[i].top) * way.bins);
      offs[i] = off < (float)kBins ? (int)off : kBins;
    }
    __syncthreads();
    constexpr int B = kBins / kPieceThreads;
    u64 own[B] = {};
    const uint32_t* h = a.bins + (int64_t)local * a.pieces * kBins;
#pragma unroll 8
    for (int i = 0; i < a.pieces; ++i) {
#pragma unroll
      for (int k = 0; k < B; ++k) {
        const int b = (int)threadIdx.x * B + k - offs[i];
        const uint32_t x = collect(h + (int64_t)i * kBins + max(b, 0));
        own[k] += b < 0 ? 0 : x;
      }
    }
    // by mass: a bin's sum is in units of 2^-16 of its least weight; bin b's begins at floor(m bins) - b, 1/32 octave each
    double sums[B], total = 0.0;
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const int b = (int)threadIdx.x * B + k;
      sums[k] = (double)own[k];
      if (by_mass)
        sums[k] *= power(fmin(0.0, ((double)row_bin - b) / kBinsPerOctave - (double)m * way.c), a.unit - 16);
      total += sums[k];
    }
    double under = total;
    running(under, dscratch);
    under -= total;
    if (threadIdx.x == 0) found = found_piece = -1;
    __syncthreads();
    // the bins at which the wanted may be reached: sums are within `off` (2^-17 and the rounding of z bins, whose 2^-24
    // of a bin are 1/46 of a weight; twice that), so the first is sought with sums that much larger, the last smaller
    const double want = by_mass ? p.top_p * whole : (double)p.top_k, off = by_mass ? 2e-5 + fabsf(row_bin) * 2.6e-9 : 0.0;
    int first_bin = kBins, last_bin = kBins;
#pragma unroll
    for (int k = 0; k < B; ++k) {
      under += sums[k];
      const int b = threadIdx.x * B + k;
      if (under * (1.0 + off) >= want) first_bin = min(first_bin, b);
      if (under * (1.0 - off) >= want) last_bin = min(last_bin, b);
    }
    // (a wavefront at a time: as few steps on one address as there are wavefronts)
    const u64 reached = __ballot(first_bin < kBins), passed = __ballot(last_bin < kBins);
    if (reached && pc.lane == __builtin_ctzll(reached)) atomicMin((unsigned*)&found, (unsigned)first_bin);
    if (passed && pc.lane == __builtin_ctzll(passed)) atomicMin((unsigned*)&found_piece, (unsigned)last_bin);
    __syncthreads();
    const int b = found, b_last = found_piece;
    if (b_last < 0)
      mode = kLeft;
    else
      hi_bin = row_bin - (float)b, lo_bin = row_bin - (float)b_last;
    if (count && p.top_k <= kListCount) hi_bin = INFINITY, mode = mode == kLeft ? kLeft : kListed;
  }
  if (mode != kLeft && way.by_share && mode != kListed) {
    // the least weight's bin, by a formula that may be off by one
    const float s = floorf((float)(((double)m * way.c + log2(p.min_p)) * kBinsPerOctave));
    if (lo_bin > s + 1.f) {
    } else if (hi_bin < s - 1.f) {
      lo_bin = s - 1.f, hi_bin = s + 1.f;
    } else {
      lo_bin = fminf(lo_bin, s - 1.f), hi_bin = fmaxf(hi_bin, s + 1.f);
    }
  }
  // (a top_k that leaves all: nothing is cut by count)
  if (mode == kLeft || (mode == kSums && lo_bin == -INFINITY)) {
    if (threadIdx.x == 0) state.mode = kDone;
    choose_row<BF>(a, r, *(Shared*)lds);
    return;
  }
  if (threadIdx.x == 0) state = RowState{m, lo_bin, hi_bin, mode, live, 0, whole};
}

// The gathering launch: 21 us for the same rows, 7 of them for the piece (loaded again, its list, the weights above it) and
// 7 for the join.
template <bool BF>
__global__ __launch_bounds__(kPieceThreads, 4) void gather_kernel(const ChooseArgs a) {
  constexpr int N = RowOf<BF>::N, V = Piece<BF>::V, W = kPieceWaves;
  __shared__ __attribute__((aligned(16))) u64 lds[2 * kList];
  static_assert(sizeof(Shared) <= sizeof(lds), "a row alone");
  u64 *keys = lds, *upto = lds + kList;
  __shared__ u64 scratch[W], extra[kPieceThreads];
  __shared__ u64 batch_sums[V * W];
  __shared__ int counts[W], listed, over_listed, base, found;
  __shared__ u64 inner;
  const int rec = blockIdx.x, local = rec / a.pieces, piece = rec - local * a.pieces;
  const RowState st = a.state[local];
  if (st.mode != kListed && st.mode != kSums) return;
  const int64_t r = a.row0 + local;
  const Sampling p = a.each ? a.each[r] : a.all;
  const float u = a.uniform[r];
  const Way way(p, u, a.vocab);
  Piece<BF> pc(a, r, piece);
  static_assert(V * W == 64, "a lane for each of a piece's sums");
  if (threadIdx.x == 0) listed = over_listed = 0;
  if (threadIdx.x < V * W) batch_sums[threadIdx.x] = 0;
  __syncthreads();
  const auto w_of = [&](float z) { return weight(((double)z - st.m) * way.c, a.unit); };
  const auto is_above = [&](float z) { return floorf(z * way.bins) > st.hi_bin; };
  u64 sum = 0;
  int above = 0, here = 0;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < N && i < pc.batches; ++j) {
      const float z = pc.at(i, j), b = floorf(z * way.bins);
      if (z > -INFINITY && b >= st.lo_bin) {
        if (b <= st.hi_bin)
          ++here;
        else
          ++above;
      }
    }
  // The weights above the list.  Few entries of a row are there as a rule, but some in nearly every wavefront: they are put
  // next to each other first (200 rows of 151936 in bf16, top-p 0.9: 133 us for both launches, 141 by batches).
  if (st.mode == kSums) {
    if (above > 0) {
      int at = atomicAdd(&over_listed, above);
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N && i < pc.batches; ++j) {
          const float z = pc.at(i, j);
          if (!is_above(z)) continue;
          if (at < kList) upto[at] = (u64)(i * W + pc.wave) << 32 | __float_as_uint(z);
          ++at;
        }
    }
    __syncthreads();
    if (over_listed <= kList) {
      for (int i = threadIdx.x; i < over_listed; i += kPieceThreads)
        atomicAdd(&batch_sums[upto[i] >> 32], w_of(__uint_as_float((uint32_t)upto[i])));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (i >= pc.batches) break;
        u64 part = 0;
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (is_above(pc.at(i, j))) part += w_of(pc.at(i, j));
        part = wave_sum(part);
        if (pc.lane == 0) batch_sums[i * W + pc.wave] = part;
      }
    }
  }
  list_entries(pc, here, [&](float z) {
    const float b = floorf(z * way.bins);
    return z > -INFINITY && b >= st.lo_bin && b <= st.hi_bin;
  }, keys, &listed);
  if (st.mode == kSums) {
    above = wave_sum(above);
    if (pc.lane == 0) counts[pc.wave] = above;
    __syncthreads();
    if (pc.wave == 0) {  // V * W of them
      sum = pc.lane < a.batches * W ? batch_sums[pc.lane] : 0;
      if (pc.lane < a.batches * W) publish(a.subs + (int64_t)rec * V * W + pc.lane, sum);
      sum = wave_sum(sum);
    }
  }
  __syncthreads();
  PieceState& mine = a.piece[rec];
  int32_t* list_n = a.list_n + local * kCounterStride;
  u64* list = a.list + (int64_t)local * kList;
  if (threadIdx.x == 0) {
    if (st.mode == kSums) {
      above = 0;
      for (int i = 0; i < W; ++i) above += counts[i];
      publish(&mine.sum, sum);
      publish(&mine.live, above);
    }
    base = listed ? __hip_atomic_fetch_add(list_n, listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < min(listed, kList); i += kPieceThreads)
    if (base < kList - i) publish(list + base + i, keys[i]);
  if (!arrive(a.arrived + local * kCounterStride, a.pieces)) return;

  // ---- the row ----
  const int n = collect(list_n);
  __syncthreads();
  if (threadIdx.x == 0) publish(list_n, (int32_t)0);
  if (n > kList || u == 0.f) {
    choose_row<BF>(a, r, *(Shared*)lds);
    return;
  }
  rank_list(keys, list, n);
  // what lies above the list
  u64 over = 0;
  int over_count = 0;
  const PieceState* all = a.piece + (int64_t)local * a.pieces;
  const int per = (a.pieces + kPieceThreads - 1) / kPieceThreads, from_piece = min(a.pieces, (int)threadIdx.x * per),
            to_piece = min(a.pieces, ((int)threadIdx.x + 1) * per);
  if (st.mode == kSums) {
    u64 x = 0;
    int c = 0;
    for (int i = from_piece; i < to_piece; ++i) x += collect(&all[i].sum), c += collect(&all[i].live);
    over = running(x, scratch);
    over_count = running(c, counts);
  }
  const Kept kept = cut_list(p, way, u, a.unit, st.m, way.by_count && p.top_k < st.live, st.whole, over, over_count, keys, upto,
                             n, w_of, scratch, counts);
  if (threadIdx.x == 0) found = 0;
  __syncthreads();
  if (st.mode == kListed) {
    find_listed(kept, keys, upto, scratch, &found);
  } else {
    // pieces (by ranges, a thread each), then a piece's wavefronts' batches, then entries, each with the kept entries
    // of the list in them
    const u64 cut = kept.count > 0 ? keys[kept.count - 1] : ~0ull;
    const int entries = a.batches * kPieceThreads * N;  // of a piece
    const auto piece_of = [&](int e) { return (e + pc.row.off) / entries; };
    const auto add_list = [&](auto place) {  // adds the list's weights to extra[place(entry)] (-1: none)
      extra[threadIdx.x] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < kept.count; i += kPieceThreads) {
        const int at = place(index_of(keys[i]));
        if (at >= 0) atomicAdd(&extra[at], upto[i]);
      }
      __syncthreads();
    };
    add_list([&](int e) { return piece_of(e) / per; });
    u64 x = extra[threadIdx.x];
    for (int i = from_piece; i < to_piece; ++i) x += collect(&all[i].sum);
    u64 ahead = x;
    running(ahead, scratch);
    ahead -= x;
    if (x > 0 && ahead <= kept.target && ahead + x > kept.target) {
      int i = from_piece;
      for (; i < to_piece - 1; ++i) {
        u64 y = collect(&all[i].sum);
        for (int k = 0; k < kept.count; ++k)
          if (piece_of(index_of(keys[k])) == i) y += upto[k];
        if (ahead + y > kept.target) break;
        ahead += y;
      }
      found = i, inner = kept.target - ahead;
    }
    __syncthreads();
    const int at = found;
    u64 want = inner;
    __syncthreads();
    add_list([&](int e) { return piece_of(e) == at ? ((e + pc.row.off) / (64 * N)) % (a.batches * W) : -1; });
    const u64* subs = a.subs + ((int64_t)local * a.pieces + at) * V * W;
    const u64 part = (int)threadIdx.x < a.batches * W ? collect(subs + threadIdx.x) + extra[threadIdx.x] : 0;
    u64 sums = part;
    running(sums, scratch);
    if (part > 0 && sums > want && sums - part <= want) found = threadIdx.x, inner = sums - part;
    __syncthreads();
    want -= inner;
    const int from = (at * a.batches * W + found) * 64;
    __syncthreads();
    find_entry<BF>(pc.row, from, want,
                   [&](float z, int i) -> u64 {
                     if (!(z > -INFINITY)) return 0;
                     const float b = floorf(z * way.bins);
                     const bool in = b > st.hi_bin || (b >= st.lo_bin && kept.count > 0 && key_of(z, i) >= cut);
                     return in ? w_of(z) : 0;
                   },
                   scratch, &found);
  }
  if (threadIdx.x == 0) {
    const double y = ((double)Elem<BF>::load(pc.row.base, found) - st.m) * way.c;
    write_token(a, r, found, log_share(y, kept.whole, a.unit), over_count + kept.count);
  }
}

// A small top-k in one launch: an entry of the first top_k of a row is one of the first top_k of its piece, so
// among those from the bin on that holds the top_k-th largest of the piece's threads' maxima (kBins bins as above).
// These go into the row's list, which the last piece ranks and cuts.
// 16 rows of 151936 in bf16, top-k 50 and top-p: 17 us in 19 pieces a row, bound by the chain of a piece (its batch,
// maximum, bins, list) and of the join (list, ranking, cut), not by the 1 us of reading; 35 in two launches.
template <bool BF>
__global__ __launch_bounds__(kPieceThreads, 4) void top_kernel(const ChooseArgs a) {
  constexpr int N = RowOf<BF>::N, V = Piece<BF>::V, W = kPieceWaves;
  __shared__ __attribute__((aligned(16))) u64 lds[2 * kList];
  u64 *keys = lds, *upto = lds + kList;
  int* bins = (int*)upto;
  __shared__ u64 scratch[W];
  __shared__ float tops[W];
  __shared__ int counts[W], listed, found;
  const int rec = blockIdx.x, local = rec / a.pieces, piece = rec - local * a.pieces;
  const int64_t r = a.row0 + local;
  const Sampling& p = a.all;
  const float u = a.uniform[r];
  const Way way(p, u, a.vocab);
  if (!way.ok) {
    if (piece == 0 && threadIdx.x == 0) write_token(a, r, -1, NAN, 0);
    return;
  }
  Piece<BF> pc(a, r, piece);
  for (int i = threadIdx.x; i < kBins; i += kPieceThreads) bins[i] = 0;
  if (threadIdx.x == 0) listed = 0, found = kBins;
  float top = -INFINITY;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < N && i < pc.batches; ++j) {
      odd |= !(pc.at(i, j) < INFINITY);
      top = fmaxf(top, pc.at(i, j));
    }
  float m = top;
  for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i));
  if (pc.lane == 0) tops[pc.wave] = m;
  odd = __syncthreads_or(odd);
  m = tops[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, tops[i]);
  float row_bin = floorf(m * way.bins);
  const auto bin_of = [&](float z) {  // below the bins, and where they are no numbers: the last
    const float b = row_bin - floorf(z * way.bins);
    return b < (float)(kBins - 1) ? (int)b : kBins - 1;
  };
  // the first bin with which bins[] has top_k, kBins where it has fewer (found is that before)
  const auto first_bin = [&] {
    __syncthreads();
    constexpr int B = kBins / kPieceThreads;
    int own = 0;
#pragma unroll
    for (int k = 0; k < B; ++k) own += bins[threadIdx.x * B + k];
    int upto_here = own;
    running(upto_here, counts);
    if (upto_here >= p.top_k && upto_here - own < p.top_k) {
      int b = threadIdx.x * B, n = upto_here - own;
      while ((n += bins[b]) < p.top_k) ++b;
      found = b;
    }
    __syncthreads();
    return found;
  };
  if (top > -INFINITY) atomicAdd(&bins[bin_of(top)], 1);
  int least = first_bin();
  if (least == kBins) {  // fewer threads with an entry than top_k (a piece at the end of a row): by all entries
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kPieceThreads) bins[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N && i < pc.batches; ++j)
        if (pc.at(i, j) > -INFINITY) atomicAdd(&bins[bin_of(pc.at(i, j))], 1);
    least = first_bin();
  }
  // each piece has room for `room` keys; kOdd and kMany, above all keys, say that the row has none, and that there is none
  constexpr u64 kOdd = ~0ull, kMany = ~0ull - 1;
  const int room = kList / a.pieces;
  if (!odd) {
    const auto in = [&](float z) { return z > -INFINITY && bin_of(z) <= least; };
    int here = 0;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N && i < pc.batches; ++j) here += in(pc.at(i, j));
    list_entries(pc, here, in, keys, &listed);
  }
  __syncthreads();
  u64* list = a.list + (int64_t)local * kList;
  for (int i = threadIdx.x; i < room; i += kPieceThreads)
    publish(list + piece * room + i, odd ? kOdd : listed > room ? kMany : i < listed ? keys[i] : 0ull);
  if (!arrive(a.arrived + local * kCounterStride, a.pieces)) return;

  // ---- the row ----
  const int n = room * a.pieces;
  // the list once more from the bin on that holds the top_k-th of all
  constexpr int P = kList / kPieceThreads;
  u64 key[P], best = 0;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int i = k * kPieceThreads + (int)threadIdx.x;
    key[k] = i < n ? collect(list + i) : 0;
    best = max(best, key[k]);
  }
  for (int i = threadIdx.x; i < kBins; i += kPieceThreads) bins[i] = 0;
  for (int i = 1; i < 64; i <<= 1) best = max(best, __shfl_xor(best, i));
  __syncthreads();
  if (pc.lane == 0) scratch[pc.wave] = best;
  if (threadIdx.x == 0) listed = 0, found = kBins;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) best = max(best, scratch[i]);
  if (best == 0 || best == kOdd) {
    if (threadIdx.x == 0) write_token(a, r, -1, NAN, 0);
    return;
  }
  if (best == kMany || u == 0.f) {
    choose_row<BF>(a, r, *(Shared*)lds);
    return;
  }
  m = value_of(best);
  row_bin = floorf(m * way.bins);
#pragma unroll
  for (int k = 0; k < P; ++k)
    if (key[k]) atomicAdd(&bins[bin_of(value_of(key[k]))], 1);
  const int cut = first_bin();
#pragma unroll
  for (int k = 0; k < P; ++k)
    if (key[k] && bin_of(value_of(key[k])) <= cut) keys[atomicAdd(&listed, 1)] = key[k];
  __syncthreads();
  const int few = listed;
  int size = 64;
  while (size < few) size <<= 1;
  if (few > kPieceThreads)
    for (int i = few + (int)threadIdx.x; i < size; i += kPieceThreads) keys[i] = 0;
  sort_keys(keys, few, size);
  const auto w_of = [&](float z) { return weight(((double)z - m) * way.c, a.unit); };
  const Kept kept = cut_list(p, way, u, a.unit, m, true, 0.0, 0, 0, keys, upto, few, w_of, scratch, counts);
  find_listed(kept, keys, upto, scratch, &found);
  if (threadIdx.x == 0) {
    const double y = ((double)Elem<BF>::load(pc.row.base, found) - m) * way.c;
    write_token(a, r, found, log_share(y, kept.whole, a.unit), kept.count);
  }
}

// The first place of x > target among the threads with own > 0, or the last of these where rounding leaves none; -1: no
// own > 0.  x: running sums.
__device__ __forceinline__ int first_above(double x, double own, double target, int* low, int* high) {
  __syncthreads();
  if (threadIdx.x == 0) *low = INT32_MAX, *high = -1;
  __syncthreads();
  const u64 some = __ballot(own > 0.0), here = __ballot(own > 0.0 && x > target);
  const int lane = threadIdx.x & 63;
  if (here && lane == __builtin_ctzll(here)) atomicMin(low, (int)threadIdx.x);
  if (some && lane == 63 - __builtin_clzll(some)) atomicMax(high, (int)threadIdx.x);
  __syncthreads();
  return *low < INT32_MAX ? *low : *high;
}

// The whole distribution, read once: the sums of pieces, of their wavefronts' batches and at last of 64 vectors narrow
// the place down.  Sums are doubles here, added in an order that sizes and alignment fix.
// 512 rows of 151936 in bf16: 101 us, 1.5 TB/s: bound by the weights in double, some 40 us of them, and by the chain of
// a piece in front of and behind them (138 in two launches).
template <bool BF>
__global__ __launch_bounds__(kPieceThreads, 4) void whole_kernel(const ChooseArgs a) {
  constexpr int N = RowOf<BF>::N, V = Piece<BF>::V, W = kPieceWaves;
  __shared__ __attribute__((aligned(16))) char lds[sizeof(Shared)];
  __shared__ double scratch[W];
  __shared__ float tops[W];
  __shared__ int lives[W], low, high;
  __shared__ double inner;
  const int rec = blockIdx.x, local = rec / a.pieces, piece = rec - local * a.pieces;
  const int64_t r = a.row0 + local;
  const float u = a.uniform[r];
  const Way way(a.all, u, a.vocab);
  if (!way.ok) {
    if (piece == 0 && threadIdx.x == 0) write_token(a, r, -1, NAN, 0);
    return;
  }
  Piece<BF> pc(a, r, piece);
  float m = -INFINITY;
  int live = 0;
  uint32_t some = 0;  // batches with an entry that is not masked
  bool odd = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int before = live;
#pragma unroll
    for (int j = 0; j < N && i < pc.batches; ++j) {
      const float z = pc.at(i, j);
      odd |= !(z < INFINITY);
      m = fmaxf(m, z);
      live += z > -INFINITY;
    }
    some |= live > before ? 1u << i : 0u;
  }
  for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i)), live += __shfl_xor(live, i);
  if (pc.lane == 0) tops[pc.wave] = m, lives[pc.wave] = live;
  odd = __syncthreads_or(odd);
  m = tops[0], live = lives[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, tops[i]), live += lives[i];
  double sum = 0.0;
  double* subs = (double*)a.subs + (int64_t)rec * V * W;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (i >= pc.batches) break;
    double part = 0.0;
    // A masked entry next to others adds 2^-200 of the largest weight, which its batch's sum may hold: an entry that is not
    // masked is there to take the place.  A batch of masked entries alone must not have one, so it weighs 0: a target that
    // is exactly the sum ahead of it (0 here) would stop at anything more.
    if (m > -INFINITY && !odd && __any(some >> i & 1)) {
#pragma unroll
      for (int j = 0; j < N; ++j) part += power(((double)Elem<BF>::get(pc.x[i], j) - m) * way.c, 0);
      part = wave_sum(part);
    }
    sum += part;
    if (pc.lane == 0) publish(subs + i * W + pc.wave, part);
  }
  if (pc.lane == 0) scratch[pc.wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    PieceState& mine = a.piece[rec];
    sum = 0.0;
    for (int i = 0; i < W; ++i) sum += scratch[i];
    publish(&mine.top, odd ? NAN : m);
    publish(&mine.live, live);
    publish(&mine.sum, (u64)__double_as_longlong(sum));
  }
  if (!arrive(a.arrived + local * kCounterStride, a.pieces)) return;

  // ---- the row ----
  const PieceState* all = a.piece + (int64_t)local * a.pieces;
  const int per = (a.pieces + kPieceThreads - 1) / kPieceThreads, from_piece = min(a.pieces, (int)threadIdx.x * per),
            to_piece = min(a.pieces, from_piece + per);
  m = -INFINITY, live = 0, odd = false;
  for (int i = from_piece; i < to_piece; ++i) {
    const float t = collect(&all[i].top);
    odd |= t != t;
    m = fmaxf(m, t);
    live += collect(&all[i].live);
  }
  for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i)), live += __shfl_xor(live, i);
  if (pc.lane == 0) tops[pc.wave] = m, lives[pc.wave] = live;
  odd = __syncthreads_or(odd);
  m = tops[0], live = lives[0];
#pragma unroll
  for (int i = 1; i < W; ++i) m = fmaxf(m, tops[i]), live += lives[i];
  if (odd || live == 0) {
    if (threadIdx.x == 0) write_token(a, r, -1, NAN, 0);
    return;
  }
  if (u == 0.f) {  // the first entry of any weight at all
    choose_row<BF>(a, r, *(Shared*)lds);
    return;
  }
  const auto sum_of = [&](int i) {  // of a piece, in units of the row's largest weight
    const float t = collect(&all[i].top);
    return t > -INFINITY ? __longlong_as_double((long long)collect(&all[i].sum)) * power(((double)t - m) * way.c, 0) : 0.0;
  };
  double own = 0.0;
  for (int i = from_piece; i < to_piece; ++i) own += sum_of(i);
  double upto = own;
  const double whole = running(upto, scratch), target = (double)u * whole;
  const int mine = first_above(upto, own, target, &low, &high);
  if ((int)threadIdx.x == mine) {
    double ahead = upto - own, x = 0.0;
    int i = from_piece;  // of the pieces with any weight (one has: own > 0), the last if rounding leaves none
    for (int j = from_piece; j < to_piece; ++j) {
      const double y = sum_of(j);
      if (y == 0.0) continue;
      ahead += x, x = y, i = j;
      if (ahead + x > target) break;
    }
    high = i;
    inner = fmax(0.0, target - ahead);
  }
  __syncthreads();
  const int at = high;
  const float t = collect(&all[at].top);
  double want = inner / power(((double)t - m) * way.c, 0);  // in the piece's units
  const double* of = (const double*)a.subs + ((int64_t)local * a.pieces + at) * V * W;
  const double part = (int)threadIdx.x < a.batches * W ? collect(of + threadIdx.x) : 0.0;
  double sums = part;
  running(sums, scratch);
  const int sub = first_above(sums, part, want, &low, &high);
  if ((int)threadIdx.x == sub) inner = sums - part;
  __syncthreads();
  want -= inner;
  const int i = pc.row.index((at * a.batches * W + sub) * 64, 0) + (int)threadIdx.x;
  double w = 0.0;
  if (threadIdx.x < 64 * N && i >= 0 && i < a.vocab) {
    const float z = Elem<BF>::load(pc.row.base, i);
    if (z > -INFINITY) w = power(((double)z - t) * way.c, 0);
  }
  sums = w;
  running(sums, scratch);
  if ((int)threadIdx.x == first_above(sums, w, want, &low, &high)) {
    const double y = ((double)Elem<BF>::load(pc.row.base, i) - m) * way.c;
    write_token(a, r, i, y * 0.69314718055994530942 - log(whole), live);
  }
}

}  // namespace

// Launches go over as many rows at a time as the records hold.
hipError_t launch_choose(ChooseArgs& a, bool bf16, hipStream_t stream) {
  a.unit = 62;
  while ((int64_t(1) << (62 - a.unit)) < a.vocab) --a.unit;
  a.unit = std::min(a.unit, 50);
  a.batches = choose_batches(a.rows, a.vocab, bf16);
  a.pieces = choose_pieces(a.vocab, a.batches, bf16);
  const int per_launch = choose_rows(a.pieces);
  const infs_sampling& p = a.all;
  const bool whole = !a.each && (p.top_k == 0 || p.top_k >= a.vocab) && (p.top_p == 0.0 || p.top_p == 1.0) && p.min_p == 0.0;
  // lists of all pieces' first top_k, with room for what else lies in their last bins
  bool top = !a.each && p.top_k > 0 && p.top_k < a.vocab && p.top_k <= kPieceThreads / 2;
  // (for few long rows that takes pieces of more entries: one row of 243428, top-k 64: 48 us in two launches of 60 pieces,
  // 17 in one of 30; where the largest are still too many, the two launches keep them, since their joins go by pieces: one
  // row of 151936 in fp32, top-k 250: 37 us in 10 pieces, 61 in 75)
  for (; top && (int64_t)p.top_k * a.pieces > kList / 2; a.pieces = choose_pieces(a.vocab, a.batches, bf16)) {
    if (a.batches < kPieceVectors)
      ++a.batches;
    else
      top = false;
  }
  const int rows = a.rows;
  for (a.row0 = 0; a.row0 < rows; a.row0 += per_launch) {
    const int n = std::min(per_launch, rows - a.row0);
    const dim3 grid((unsigned)n * a.pieces), block(kPieceThreads);
    if (whole) {
      hipLaunchKernelGGL(bf16 ? whole_kernel<true> : whole_kernel<false>, grid, block, 0, stream, a);
    } else if (top) {
      hipLaunchKernelGGL(bf16 ? top_kernel<true> : top_kernel<false>, grid, block, 0, stream, a);
    } else {
      hipLaunchKernelGGL(bf16 ? weigh_kernel<true> : weigh_kernel<false>, grid, block, 0, stream, a);
      hipLaunchKernelGGL(bf16 ? gather_kernel<true> : gather_kernel<false>, grid, block, 0, stream, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace infs
