// Scores of tokens: log probabilities, entropies and most probable entries of
// rows of logits, and the gradient of the former two.
//
// With m = max z, y_j = (z_j - m) / T and S = sum e^y_j:  log p_j = y_j - ln S and
// entropy = ln S - (sum e^y_j y_j) / S.  A part of a row is (m, S, W = sum e^y y),
// taken in one pass around a running maximum; two parts join at the larger
// maximum as S = sum_i S_i e^(d_i), W = sum_i (W_i + S_i d_i) e^(d_i) with d_i =
// (m_i - m) / T.  Exponents are in units of log 2 (y2 = y log2 e).  Masked entries
// (-inf) and far ones have e^y = 0; y is held above -1000 where it is multiplied,
// so that 0 * -inf does not arise.  The running maximum starts at the lowest
// finite number, so that a difference of two infinities arises from +inf alone,
// which makes S a NaN, as a NaN does.
#include "ops.h"

#include <float.h>

#include <algorithm>

namespace infs {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kThreads = kBlockThreads;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kFar = -1000.f;  // 2^kFar is 0

template <bool BF>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  if constexpr (BF)
    return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
  else
    return ((const float*)p)[i];
}
template <bool BF>
__device__ __forceinline__ void store1(void* p, int64_t i, float x) {
  if constexpr (BF)
    ((uint16_t*)p)[i] = __builtin_bit_cast(uint16_t, (__bf16)x);
  else
    ((float*)p)[i] = x;
}

struct Part {
  float m, s, w;
};
__device__ __forceinline__ Part empty_part() { return Part{-FLT_MAX, 0.f, 0.f}; }

// Order of alternatives as one number: by value, then by the lower index; 0: none.
__device__ __forceinline__ unsigned long long key_of(float x, int i) {
  if (!(x > -__builtin_huge_valf())) return 0;
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 counts as 0
  const uint32_t o = (b >> 31) ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (uint32_t)~i;
}
__device__ __forceinline__ int key_id(unsigned long long k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(unsigned long long k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o);
}

// ---- the forward pass ----------------------------------------------------------
//
// A row is read once, 16 bytes a lane and load.  Loads go by aligned vectors of
// N elements: vector v covers elements v N - lead .. of the row, lead the elements
// by which the row's start lies behind a 16-byte boundary; the first and the last
// vector of a row may be in part outside it and are then read by elements, what is
// outside counting as masked.  W wavefronts take a row (a work-group, or one of its
// wavefronts where rows are many and short) in batches of kUnroll vectors a lane,
// every lane around its own running maximum.
//
// Few rows are cut into pieces of whole batches, a work-group each; the pieces of a
// row are joined by the work-group that finishes last, always in the same order.
//
// Many rows are bound by memory: 2048 x 151936 bf16 takes 111 us, 5.6 TB/s (loads past the
// caches; 9 % more through them).  An element costs about ten operations of the vector
// unit (the exponential four), 15 would be all its time at that rate, so that
// alternatives, which keep the batch's elements beside its exponentials, bind that
// unit: 13 % more with 20 of them.  16 rows, each cut into 19 pieces of one batch, take 9 us:
// 2.2 thousand cycles until the batch is there (behind the row's token and that token's
// logit, which every piece loads first), 6 for its sums and candidates, 2 until a
// piece has arrived, 6 for the join, and the launch.
//
// kUnroll: 8 vectors a lane are 5 % faster on 2048 rows and a third slower on 301 x 50257
// fp32 and on short rows; loading a batch ahead is 5 % faster on 2048 rows and 10 to 25 %
// slower below.
constexpr int kUnroll = 4;
constexpr int kBatch = kThreads * kUnroll;  // vectors of a batch of a work-group
constexpr int kMaxPieces = kScoreMaxPieces;
constexpr int kWaveKeys = INFS_SCORE_MAX_TOP + 64 * 8;  // candidates a wavefront holds: a vector a lane beside the best
constexpr int kKeptKeys = 64;                           // most it hands on
constexpr int kFewLanes = 8;  // lanes with candidates in a batch that do not move a wavefront's bound
static_assert(INFS_SCORE_MAX_TOP <= kKeptKeys, "candidate buffers");
constexpr int kPieceKeys = kScorePieceKeys;
static_assert(kMaxPieces <= 64, "a lane a piece");
static_assert(kPieceKeys >= INFS_SCORE_MAX_TOP && kPieceKeys <= kThreads && kMaxPieces * kPieceKeys % kThreads == 0 &&
                  kMaxPieces * kPieceKeys + 8 <= kWaves * kWaveKeys,
              "joining pieces");

template <bool BF>
struct Vec {
  static constexpr int N = BF ? 8 : 4, ES = BF ? 2 : 4;
  static __device__ __forceinline__ float get(const u32x4& v, int i) {
    if constexpr (BF) {
      const uint32_t w = v[i >> 1];
      return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
    } else {
      return __uint_as_float(v[i]);
    }
  }
  static constexpr uint32_t kMasked = BF ? 0xff80ff80u : 0xff800000u;
};

// One row's vectors.
template <bool BF>
struct RowReader {
  using V = Vec<BF>;
  const char* at;     // vector 0
  const char* row;    // element 0
  int lead, vocab, count;  // elements before the row in vector 0; elements; vectors
  int lo, hi;         // vectors wholly inside the row
  __device__ RowReader(const void* logits, int64_t offset, int n) : vocab(n) {
    row = (const char*)logits + offset * V::ES;
    lead = (int)((uintptr_t)row / V::ES % V::N);
    at = row - lead * V::ES;
    count = (lead + n + V::N - 1) / V::N;
    lo = lead > 0;
    hi = (lead + n) / V::N;
  }
  // Vectors first + L u + lane of [first, end), L lanes: all loads at once, each inside the row.
  template <int L>
  __device__ __forceinline__ void load(int first, int end, u32x4 (&x)[kUnroll]) const {
    const int v0 = first + (int)threadIdx.x % L;
    if (first >= lo && first + L * kUnroll <= min(end, hi)) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        x[u] = __builtin_nontemporal_load((const u32x4*)(at + (int64_t)(v0 + u * L) * 16));
      return;
    }
    if (lo < hi) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) x[u] = *(const u32x4*)(at + (int64_t)min(max(v0 + u * L, lo), hi - 1) * 16);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int v = v0 + u * L;
      if (v >= lo && v < min(end, hi)) continue;
      x[u] = u32x4{V::kMasked, V::kMasked, V::kMasked, V::kMasked};
      if (v >= end) continue;
      const int e0 = v * V::N - lead;
      for (int e = max(e0, 0); e < min(e0 + V::N, vocab); ++e) {
        if constexpr (BF) {
          const uint32_t b = ((const uint16_t*)row)[e];
          const int i = e - e0;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            if (w == i >> 1) x[u][w] = (i & 1) ? (x[u][w] & 0xffffu) | (b << 16) : (x[u][w] & 0xffff0000u) | b;
        } else {
#pragma unroll
          for (int w = 0; w < 4; ++w)
            if (w == e - e0) x[u][w] = ((const uint32_t*)row)[e];
        }
      }
    }
  }
};

// Reductions over a wavefront without LDS: within rows of 16 lanes by lane permutations, then
// each row's total to the next row and the lower half's to the upper; lane 63 ends with all of it.
template <int CTRL, int ROWS>
__device__ __forceinline__ float lanes(float old, float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float last_lane(float x) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, lanes<0xB1, 0xF>(x, x));   // quad_perm [1,0,3,2]
  x = fmaxf(x, lanes<0x4E, 0xF>(x, x));   // quad_perm [2,3,0,1]
  x = fmaxf(x, lanes<0x141, 0xF>(x, x));  // row_half_mirror
  x = fmaxf(x, lanes<0x140, 0xF>(x, x));  // row_mirror
  x = fmaxf(x, lanes<0x142, 0xA>(x, x));  // row_bcast:15 into rows 1 and 3
  x = fmaxf(x, lanes<0x143, 0xC>(x, x));  // row_bcast:31 into rows 2 and 3
  return last_lane(x);
}
__device__ __forceinline__ float wave_sum(float x) {
  x += lanes<0xB1, 0xF>(0.f, x);
  x += lanes<0x4E, 0xF>(0.f, x);
  x += lanes<0x141, 0xF>(0.f, x);
  x += lanes<0x140, 0xF>(0.f, x);
  x += lanes<0x142, 0xA>(0.f, x);
  x += lanes<0x143, 0xC>(0.f, x);
  return last_lane(x);
}
// A part around another maximum (m >= p.m).
__device__ __forceinline__ Part around(const Part& p, float m, float c) {
  const float d = fmaxf((p.m - m) * c, kFar), f = __builtin_amdgcn_exp2f(d);
  return Part{m, p.s * f, (p.w + p.s * d) * f};
}
__device__ __forceinline__ Part wave_join(const Part& p, float c) {
  const Part q = around(p, wave_max(p.m), c);
  return Part{q.m, wave_sum(q.s), wave_sum(q.w)};
}

__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o); }

// The k-th largest of the lanes' 16-bit values: bit by bit, by counting lanes.
__device__ __forceinline__ uint32_t kth_largest(uint32_t o, int k) {
  uint32_t t = 0;
#pragma unroll
  for (uint32_t bit = 0x8000u; bit > 0; bit >>= 1)
    if (__popcll(__ballot(o >= (t | bit))) >= k) t |= bit;
  return t;
}
// The largest of a lane's values in the four wavefronts: 64 groups of the work-group's threads.
// (The k-th largest group maximum lets few more elements through than the k-th of all threads.)
// Two calls in a row need two buffers.
__device__ __forceinline__ uint32_t columns(uint32_t o, uint32_t* shared) {
  shared[threadIdx.x] = o;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  return max(max(shared[lane], shared[64 + lane]), max(shared[128 + lane], shared[192 + lane]));
}

// The most probable entries a wavefront has seen, as a superset: every element not
// below `bound`.  base is a value that at least k of the elements seen so far reach: the
// k-th largest of the lanes' running maxima (its upper 16 bits are taken, which can only
// lower it), or the k-th best when a full buffer was cut.  It rises as the wavefront
// reads on, so that few elements reach it, and a vector costs one comparison.  An
// element of a later batch has a higher index than all those and must exceed base.
// Before k elements are known base is the lowest number, which nothing need exceed.
struct Candidates {
  unsigned long long* keys;  // kWaveKeys in LDS
  int n, k;
  float base, bound;
  bool reached = false;  // k elements reach base
  // base to the k-th largest of the lanes' values, given by the upper halves of their orders.
  __device__ __forceinline__ void raise(uint32_t o) {
    base = fmaxf(base, value_of(kth_largest(o, k) << 16));  // NaN, below every number, drops out
    bound = fmaxf(bound, base);
    reached = reached || base > -FLT_MAX;  // lanes without elements count as the lowest number
  }
  // Before the elements of a later batch of a wavefront, whose largest in this lane is `largest` (of all
  // so far: lane_max).
  __device__ __forceinline__ void next_batch(float largest, float lane_max) {
    if (__popcll(__ballot(largest >= bound)) > kFewLanes) raise(order_of(lane_max) >> 16);
  }
  // An element of a later batch must exceed base.
  __device__ __forceinline__ void end_batch() {
    if (reached) bound = fmaxf(bound, above(base));
  }
  // The next larger number.
  static __device__ __forceinline__ float above(float x) {
    const uint32_t b = __float_as_uint(x);
    return x == 0.f ? __uint_as_float(1u) : __uint_as_float((b >> 31) ? b - 1 : b + 1);
  }
  // Cut to the k best, in order: the largest below the one before, k times.
  __device__ __forceinline__ void cut() {
    const int lane = threadIdx.x & 63;
    unsigned long long kth = ~0ull, kept = 0;
    for (int r = 0; r < min(n, k); ++r) {
      unsigned long long best = 0;
      for (int i = lane; i < n; i += 64)
        if (keys[i] < kth) best = max(best, keys[i]);
#pragma unroll
      for (int mask = 1; mask < 64; mask <<= 1) best = max(best, (unsigned long long)__shfl_xor((long long)best, mask));
      kth = best;
      if (lane == r) kept = best;
    }
    if (lane < min(n, k)) keys[lane] = kept;
    if (n >= k) {
      base = fmaxf(base, key_value(kth));
      bound = fmaxf(bound, base);
      reached = true;
    }
    n = min(n, k);
  }
  // Room for `more` (at most kWaveKeys - k).
  __device__ __forceinline__ void reserve(int more) {
    if (n + more > kWaveKeys) cut();
  }
  // The lanes' elements of vector x that reach the bound, the first of them of index e0.
  template <bool BF>
  __device__ __forceinline__ void add(const u32x4& x, int e0) {
    using V = Vec<BF>;
    reserve(64 * V::N);
    unsigned long long masks[V::N];  // all comparisons first: no branch waits for each
#pragma unroll
    for (int i = 0; i < V::N; ++i) masks[i] = __ballot(V::get(x, i) >= bound);
#pragma unroll
    for (int i = 0; i < V::N; ++i) {
      if (masks[i] == 0) continue;
      const uint32_t lo = (uint32_t)masks[i], hi = (uint32_t)(masks[i] >> 32);
      const int at = n + __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
      if (V::get(x, i) >= bound) keys[at] = key_of(V::get(x, i), e0 + i);
      n += __popcll(masks[i]);
    }
  }
};

template <int W>
__device__ __forceinline__ void row_sync() {
  if constexpr (W > 1) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Ranks by counting, by the threads of W wavefronts: the k largest of n keys to out, largest first; 0
// where fewer.  keys is kRankStep keys longer than n and aligned to 16 bytes: the reads go by whole
// steps, so that they overlap.
constexpr int kRankStep = 8;
template <int W>
__device__ __forceinline__ void rank_keys(unsigned long long* keys, int n, int k, unsigned long long* out) {
  const int t = threadIdx.x % (64 * W);
  if (t < kRankStep) keys[n + t] = 0;
  if (t < k && t >= n) out[t] = 0;
  row_sync<W>();
  for (int i = t; i < n; i += 64 * W) {
    const unsigned long long key = keys[i];
    int rank = 0;
    for (int j = 0; j < n; j += kRankStep) {
      unsigned long long x[kRankStep];
#pragma unroll
      for (int q = 0; q < kRankStep; ++q) x[q] = keys[j + q];
#pragma unroll
      for (int q = 0; q < kRankStep; ++q) rank += x[q] > key;
    }
    if (rank < k) out[rank] = key;
  }
  row_sync<W>();
}

__device__ __forceinline__ void publish(float* p, float x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void publish(unsigned long long* p, unsigned long long x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class T>
__device__ __forceinline__ T collect(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <bool BF, bool TOP, int W>
__global__ __launch_bounds__(kThreads) void score_kernel(const ScoreArgs a) {
  using V = Vec<BF>;
  constexpr int L = 64 * W;  // lanes of a row
  constexpr int kRows = kWaves / W;
  __shared__ Part parts[kWaves];
  __shared__ __attribute__((aligned(16))) unsigned long long wave_keys[TOP ? kWaves : 1][TOP ? kWaveKeys + kRankStep : 1];
  __shared__ __attribute__((aligned(16))) unsigned long long keys[TOP && W > 1 ? kWaves * kKeptKeys + kRankStep : 1];
  __shared__ unsigned long long bests[TOP ? kRows : 1][TOP ? INFS_SCORE_MAX_TOP : 1];
  __shared__ uint32_t maxima[2][TOP && W > 1 ? kThreads : 1];
  __shared__ int counts[kWaves], last;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, thread = threadIdx.x % L;
  const int piece = W > 1 ? (int)(blockIdx.x % (unsigned)a.pieces) : 0;
  const int64_t row = W > 1 ? blockIdx.x / (unsigned)a.pieces : (int64_t)blockIdx.x * kRows + wave;
  if (W == 1 && row >= a.rows) return;  // nothing waits for this wavefront
  const RowReader<BF> in(a.logits, row * a.row_stride, a.vocab);
  const float c = a.inv_t * kLog2E;
  // the given token's logit, for whoever finishes the row
  const int token = a.logprob ? a.tokens[row] : -1;
  const bool known = token >= 0 && token < a.vocab;
  const float given = known ? load1<BF>(in.row, token) : 0.f;

  Part p = empty_part();
  Candidates top{wave_keys[TOP ? wave : 0], 0, a.top_k, -FLT_MAX, -FLT_MAX};  // masked entries are below
  constexpr int kStep = L * kUnroll;
  const int begin = W > 1 ? piece * a.batches * kStep : 0, end = W > 1 ? min(begin + a.batches * kStep, in.count) : in.count;
  for (int first = begin, b = 0, raised = 0; first < end; first += kStep, ++b) {
    u32x4 x[kUnroll];
    in.template load<L>(first, end, x);
    float vm[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      vm[u] = V::get(x[u], 0);
#pragma unroll
      for (int i = 1; i < V::N; ++i) vm[u] = fmaxf(vm[u], V::get(x[u], i));
    }
    const float largest = fmaxf(fmaxf(vm[0], vm[1]), fmaxf(vm[2], vm[3]));
    p = around(p, fmaxf(p.m, largest), c);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int i = 0; i < V::N; ++i) {
        const float y = (V::get(x[u], i) - p.m) * c, e = __builtin_amdgcn_exp2f(y);
        p.s += e;
        p.w = fmaf(e, fmaxf(y, kFar), p.w);
      }
    if constexpr (TOP) {
      // the bound: from all lanes of the row at batches 0, 1, 2, 4, 8 .., else from the wavefront's
      if (W > 1 && (b & (b - 1)) == 0)
        top.raise(columns(order_of(p.m) >> 16, maxima[raised++ & 1]));
      else
        top.next_batch(largest, p.m);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (__ballot(vm[u] >= top.bound) != 0) top.template add<BF>(x[u], (first + u * L + thread) * V::N - in.lead);
      top.end_batch();
    }
  }

  // the part of the row's wavefronts
  p = wave_join(p, c);
  if constexpr (W > 1) {
    if (lane == 0) parts[wave] = p;
  }
  if constexpr (TOP) {
    if (top.n > kKeptKeys) top.cut();
    if (W > 1 && lane == 0) counts[wave] = top.n;
  }
  unsigned long long* best = bests[TOP && W == 1 ? wave : 0];
  if constexpr (W == 1) {
    if constexpr (TOP) rank_keys<1>(wave_keys[wave], top.n, a.top_k, best);
  } else {
    __syncthreads();
    Part q[kWaves];
    float m = parts[0].m;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, parts[w].m);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) q[w] = around(parts[w], m, c);
    p = Part{m, (q[0].s + q[1].s) + (q[2].s + q[3].s), (q[0].w + q[1].w) + (q[2].w + q[3].w)};
    int before = 0, found = 0;  // candidates of the wavefronts before this one, and of all
    if constexpr (TOP) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += counts[w];
        found += counts[w];
      }
      if (a.pieces == 1 || found > kPieceKeys) {
        if (lane < counts[wave]) keys[before + lane] = wave_keys[wave][lane];
        rank_keys<W>(keys, found, a.top_k, best);
      }
    }
    if (a.pieces > 1) {
      // Hand the part over, and the candidates (more than kPieceKeys: the best); the last work-group
      // of the row joins them.
      const int64_t rec = row * a.pieces + piece;
      if (threadIdx.x == 0) {
        float* to = a.part + kScorePartStride * rec;
        publish(to, p.m);
        publish(to + 1, p.s);
        publish(to + 2, p.w);
      }
      if constexpr (TOP) {
        unsigned long long* to = a.keys + rec * kPieceKeys;
        if (found > kPieceKeys) {
          if ((int)threadIdx.x < kPieceKeys) publish(to + threadIdx.x, (int)threadIdx.x < a.top_k ? best[threadIdx.x] : 0);
        } else {
          if (lane < counts[wave]) publish(to + before + lane, wave_keys[wave][lane]);
          if ((int)threadIdx.x >= found && (int)threadIdx.x < kPieceKeys) publish(to + threadIdx.x, 0);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_s_waitcnt(0);  // this thread's stores have reached the coherence point
      __syncthreads();
      if (threadIdx.x == 0) {
        int32_t* arrived = a.arrived + row * kCounterStride;
        last = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.pieces - 1;
        if (last) __hip_atomic_store(arrived, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
        counts[0] = 0;
      }
      __syncthreads();
      if (!last) return;
      constexpr int kMine = TOP ? kMaxPieces * kPieceKeys / kThreads : 1;
      unsigned long long mine[kMine];
      if constexpr (TOP) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const int at = i * kThreads + (int)threadIdx.x;
          mine[i] = at < a.pieces * kPieceKeys ? collect(a.keys + row * a.pieces * kPieceKeys + at) : 0;
        }
      }
      if (wave == 0) {
        Part t = empty_part();
        if (lane < a.pieces) {
          const float* r = a.part + kScorePartStride * (row * a.pieces + lane);
          t = Part{collect(r), collect(r + 1), collect(r + 2)};
        }
        t = wave_join(t, c);
        if (lane == 0) parts[0] = t;
      }
      if constexpr (TOP) {
        // the best of them, again by a bound that at least k reach
        unsigned long long* all = wave_keys[0];  // of all wavefronts, as one array
        unsigned long long largest = mine[0];
#pragma unroll
        for (int i = 1; i < kMine; ++i) largest = max(largest, mine[i]);
        const uint32_t least = kth_largest(columns((uint32_t)(largest >> 48), maxima[0]), a.top_k);
#pragma unroll
        for (int i = 0; i < kMine; ++i)
          if (mine[i] != 0 && (uint32_t)(mine[i] >> 48) >= least) all[atomicAdd(&counts[0], 1)] = mine[i];
        __syncthreads();
        const int kept = counts[0];
        rank_keys<W>(all, kept, a.top_k, best);
      }
      __syncthreads();
      p = parts[0];
    }
  }

  const bool none = p.s == 0.f;  // every entry masked
  const float log2_s = log2f(p.s), ln_s = none ? -__builtin_huge_valf() : log2_s * kLn2;
  if (thread == 0) {
    if (a.logprob) {
      float lp = token == -1 ? 0.f : __builtin_nanf("");
      if (known) lp = none ? -__builtin_huge_valf() : (given - p.m) * a.inv_t - ln_s;
      a.logprob[row] = lp;
    }
    if (a.entropy) a.entropy[row] = none ? 0.f : kLn2 * (log2_s - p.w / p.s);
    if (a.stats) {
      a.stats[2 * row] = none ? -__builtin_huge_valf() : p.m;
      a.stats[2 * row + 1] = ln_s;
    }
  }
  if constexpr (TOP) {
    if (thread < a.top_k) {
      const unsigned long long key = best[thread];
      const bool bad = !(p.s == p.s);
      a.top_id[row * a.top_k + thread] = key == 0 || bad ? -1 : key_id(key);
      a.top_logprob[row * a.top_k + thread] =
          bad ? __builtin_nanf("") : key == 0 ? -__builtin_huge_valf() : (key_value(key) - p.m) * a.inv_t - ln_s;
    }
  }
}

// ---- the gradient ---------------------------------------------------------------
//
// grad_j = p_j (A + B log p_j) + [j = token] C with A = -(g_lp + g_h H) / T, B = -g_h / T,
// C = g_lp / T: elements alone.  A work-group takes a batch of a row, or (W = 1) each of its
// wavefronts a row of one batch of its own.
// Loads and stores go past the caches: 2048 x 151936 bf16 takes 200 us so (6.2 TB/s), 215 us with
// loads and 228 us with both through them, and smaller calls are as fast or faster too.
template <bool BF, bool ENTROPY, int W>
__global__ __launch_bounds__(kThreads) void score_grad_kernel(const ScoreGradArgs a) {
  using V = Vec<BF>;
  constexpr int L = 64 * W;
  const int64_t row = W > 1 ? blockIdx.x / (unsigned)a.batches : (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (W == 1 && row >= a.rows) return;
  const RowReader<BF> in(a.logits, row * a.row_stride, a.vocab);
  const int first = W > 1 ? (int)(blockIdx.x % (unsigned)a.batches) * kBatch : 0;
  u32x4 x[kUnroll];
  in.template load<L>(first, in.count, x);
  char* g = (char*)a.grad + row * a.grad_row_stride * V::ES;
  const bool same = (int)((uintptr_t)g / V::ES % V::N) == in.lead;  // vectors of the two rows coincide
  const float m = a.stats[2 * row], ls2 = a.stats[2 * row + 1] * kLog2E, c = a.inv_t * kLog2E;
  const int token = a.d_logprob ? a.tokens[row] : -1;
  float g_lp = a.d_logprob && token != -1 ? a.d_logprob[row] : 0.f;
  const bool outside = token < -1 || token >= a.vocab;
  if (outside) g_lp = __builtin_nanf("");
  const float g_h = ENTROPY ? a.d_entropy[row] : 0.f;
  const float ca = -(g_lp + (ENTROPY ? g_h * a.entropy[row] : 0.f)) * a.inv_t, cb = -g_h * a.inv_t * kLn2, cc = g_lp * a.inv_t;
  const bool none = m == -__builtin_huge_valf();  // every entry masked
  const float masked = outside ? g_lp : 0.f;      // the gradient then
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int v = first + u * L + (int)threadIdx.x % L;
    if (v >= in.count) break;
    const int e0 = v * V::N - in.lead;
    float r[V::N];
#pragma unroll
    for (int i = 0; i < V::N; ++i) {
      const float y = (V::get(x[u], i) - m) * c - ls2, p = __builtin_amdgcn_exp2f(y);
      r[i] = ENTROPY ? p * fmaf(cb, fmaxf(y, kFar), ca) : p * ca;
      if (none) r[i] = masked;
    }
    if (token >= e0 && token < e0 + V::N && !none) {
#pragma unroll
      for (int i = 0; i < V::N; ++i)
        if (e0 + i == token) r[i] += cc;
    }
    if (same && v >= in.lo && v < in.hi) {
      u32x4 w;
      if constexpr (BF) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = __builtin_bit_cast(uint16_t, (__bf16)r[2 * i]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)r[2 * i + 1]) << 16;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(r[i]);
      }
      __builtin_nontemporal_store(w, (u32x4*)(g + (int64_t)e0 * V::ES));
    } else {
#pragma unroll
      for (int i = 0; i < V::N; ++i)
        if (e0 + i >= 0 && e0 + i < a.vocab) store1<BF>(g, e0 + i, r[i]);
    }
  }
}

}  // namespace

void (*score_kernel_of(bool bf16, bool top, bool wave_rows))(const ScoreArgs) {
  static void (*const kernels[2][2][2])(const ScoreArgs) = {
      {{score_kernel<false, false, kWaves>, score_kernel<false, false, 1>},
       {score_kernel<false, true, kWaves>, score_kernel<false, true, 1>}},
      {{score_kernel<true, false, kWaves>, score_kernel<true, false, 1>},
       {score_kernel<true, true, kWaves>, score_kernel<true, true, 1>}}};
  return kernels[bf16][top][wave_rows];
}

// A wavefront a row from 2048 rows (a work-group each would be more than fit the GPU at once, 1280 to 1792
// by the kernels' registers) of up to 1024 vectors: 4096 x 1000 bf16 5.9 us, 14.1 with a work-group a row;
// 4096 x 8000 with 5 alternatives 19.9 and 22.7; but 1024 x 8000 7.8 and 6.8, with alternatives 12.6 and
// 8.7.  Otherwise as many pieces of a row as leave all work-groups
// on the GPU at once: a few more than fit would run almost alone at the end (1000 x 151936 bf16 52.6 us, 57.7
// with pieces for about 1024 work-groups whatever fits; 512 x 151936 with 20 alternatives 42.5 and 45.1;
// 600 x 20000 fp32, the other way, 12.8 and 12.1).
void plan_score(ScoreArgs& a, bool bf16) {
  const int n = bf16 ? 8 : 4;
  const bool aligned = (uintptr_t)a.logits % 16 == 0 && a.row_stride % n == 0;  // every row is
  const int64_t all = (a.vocab + (aligned ? 0 : n - 1) + n - 1) / n;            // most vectors of a row
  const int64_t batches = (all + kBatch - 1) / kBatch;
  a.wave_rows = a.rows >= kScoreWaveRows && all <= kScoreWaveVectors;
  const int64_t most = std::min<int64_t>(std::min(a.resident, kScoreMaxRecords) / a.rows, kMaxPieces);
  const int64_t pieces = std::max<int64_t>(1, std::min(most, batches));
  a.batches = (int)((batches + pieces - 1) / pieces);
  a.pieces = (int)((batches + a.batches - 1) / a.batches);
}

hipError_t launch_score(ScoreArgs& a, bool bf16, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  plan_score(a, bf16);
  const int64_t blocks = a.wave_rows ? (a.rows + kWaves - 1) / kWaves : a.rows * (int64_t)a.pieces;
  hipLaunchKernelGGL(score_kernel_of(bf16, a.top_id != nullptr, a.wave_rows), dim3((unsigned)blocks), dim3(kThreads), 0,
                     stream, a);
  return hipGetLastError();
}

hipError_t score_resident(bool bf16, bool top, int* resident) {
  int per_cu = 0, dev = 0, cus = 0;
  hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, score_kernel_of(bf16, top, false), kThreads, 0);
  if (e == hipSuccess) e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e == hipSuccess) *resident = per_cu * cus;
  return e;
}

hipError_t launch_score_grad(ScoreGradArgs& a, bool bf16, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  const int n = bf16 ? 8 : 4;
  const int64_t vectors = (a.vocab + 2 * (n - 1)) / n;  // most of a row
  // Rows of a wavefront's batch go a wavefront each where they are many: 4096 x 1000 bf16 5.9 us, 7.5 us with
  // work-groups; longer ones do not (4096 x 5003 in more batches 22.1 us, 20.0 us with work-groups).
  const bool wave_rows = a.rows >= 1024 && vectors <= 64 * kUnroll;
  a.batches = (int)((vectors + kBatch - 1) / kBatch);
  const int64_t most = kMostBlocks / a.batches;  // rows of a launch
#define INFS_GRAD(bf, h) \
  { score_grad_kernel<bf, h, kWaves>, score_grad_kernel<bf, h, 1> }
  void (*const kernels[2][2][2])(const ScoreGradArgs) = {{INFS_GRAD(false, false), INFS_GRAD(false, true)},
                                                         {INFS_GRAD(true, false), INFS_GRAD(true, true)}};
#undef INFS_GRAD
  const ScoreGradArgs all = a;
  for (int64_t r0 = 0; r0 < all.rows; r0 += most) {
    a.rows = (int32_t)std::min(most, all.rows - r0);
    a.logits = (const char*)all.logits + r0 * all.row_stride * (bf16 ? 2 : 4);
    a.grad = (char*)all.grad + r0 * all.grad_row_stride * (bf16 ? 2 : 4);
    a.tokens = all.tokens ? all.tokens + r0 : nullptr;
    a.stats = all.stats + 2 * r0;
    a.entropy = all.entropy ? all.entropy + r0 : nullptr;
    a.d_logprob = all.d_logprob ? all.d_logprob + r0 : nullptr;
    a.d_entropy = all.d_entropy ? all.d_entropy + r0 : nullptr;
    const unsigned blocks = wave_rows ? (unsigned)((a.rows + kWaves - 1) / kWaves) : (unsigned)(a.rows * (int64_t)a.batches);
    hipLaunchKernelGGL(kernels[bf16][a.d_entropy != nullptr][wave_rows], dim3(blocks), dim3(kThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace infs
