// Causal attention of packed sequences with grouped heads, and its gradient.
//
// Token t of a sequence of n queries and m keys (its queries are its last
// tokens) sees keys 0 .. t + m - n.  With s = scale q.k over the seen keys:
//   lse = ln sum e^s,   o = sum e^(s - lse) v
// and with up = d_o, D = up.o, p = e^(s - lse), ds = p (up.v - D):
//   dq = scale sum ds k,   dk = scale sum ds q,   dv = sum p up
// where the sums of dk and dv run over the queries of all heads of a group.
//
// Rows.  The queries of a KV head's group are one list of rows, row r being
// token r / hpk of head r % hpk, so a tile of rows shares every key whatever
// hpk is, and dk and dv add over the heads inside a work-group.
//
// Matrix products.  A wavefront owns 32 rows (in the kernel of dk and dv, 32
// keys) as the columns of 32 x 32 products whose other side comes out of LDS:
//   s^T = K q^T,  o^T += V^T p^T
// A lane then holds one row's scores: its maximum and sum need one exchange
// with the lane 32 further.  The result of the first product is the operand
// of the second as it is: a lane's registers 8j .. 8j+7 are keys
// {4h .. 4h+3, 8+4h .. 8+4h+3} of 16 (h: which half of the wavefront), and V^T is
// read in that order (transposed out of LDS, 8 bytes of four keys a lane).
// bf16 operands add up in fp32; p and ds are rounded to bf16 as operands
// (2^-8 relative each, as the rounding of the outputs they add up to);
// fp32 rows take fp32 products.
//
// Masked places.  A score that its row does not see is replaced, not added to,
// and rows behind a sequence hold its last one again in LDS, unseen by all.  Only a product over tokens of
// one tile, some of them unseen, can meet 0 times an infinity or NaN.  Where
// such a tile holds one (seen while it is staged), the work-group starts over
// in a second pass over its tiles, in which those elements are taken out
// of the products and added token by token to the rows that see them, 32
// elements of the result at a time (so that the pass takes no more registers than
// the first; inside the first it took those of a wavefront in four).
//
// Work-groups.  C wavefronts, of 32 rows each, share the tiles, and there are S
// such groups, which take turns with the tiles and are joined at the end: many
// columns for many rows (every byte out of L2 serves 256 of them), many splits
// where there are too few work-groups to fill the GPU, and some of both between.
// Where even 32 rows a work-group leave CUs idle, several work-groups share a
// walk over the tiles.
#include "ops.h"

#include <algorithm>
#include <type_traits>

namespace infs {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;
// Scores this far out (in powers of 2) are taken off the row's base before they are scaled, since the rounding of the
// scaled base, 2^-24 of it, is on its way to be a power by itself.
constexpr float kFar = 0x1p20f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The value of the lane 32 further (or back).
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

template <bool BF>
struct Type;
template <>
struct Type<true> {
  static constexpr int kRegs = 8;  // accumulator registers that one operand takes
  static __device__ __forceinline__ f32x16 mma(f32x16 c, u32x4 a, u32x4 b) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ u32x4 operand(const f32x16& s, int i) {
    bf16x8 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (__bf16)s[i + j];
    return __builtin_bit_cast(u32x4, r);
  }
  // slot j of 8 alone
  static __device__ __forceinline__ u32x4 only(u32x4 x, int j, bool here) {
    const uint32_t m = !here ? 0u : (j & 1) ? 0xffff0000u : 0xffffu;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] &= k == j >> 1 ? m : 0u;
    return x;
  }
  // a sign bit is set where an exponent is all ones
  static __device__ __forceinline__ uint32_t odd_bits(uint32_t x) { return (x & 0x7f807f80u) + 0x00800080u; }
  // the infinities and NaN alone
  static __device__ __forceinline__ u32x4 odd_part(u32x4 x) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      r[j] = ((x[j] & 0x7f80u) == 0x7f80u ? x[j] & 0xffffu : 0u) | ((x[j] & 0x7f800000u) == 0x7f800000u ? x[j] & 0xffff0000u : 0u);
    return r;
  }
  static __device__ __forceinline__ float dot(u32x4 x, u32x4 y) {
    float r = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r = fmaf(__uint_as_float(x[j] << 16), __uint_as_float(y[j] << 16), r);
      r = fmaf(__uint_as_float(x[j] & 0xffff0000u), __uint_as_float(y[j] & 0xffff0000u), r);
    }
    return r;
  }
};
template <>
struct Type<false> {
  static constexpr int kRegs = 4;
  static __device__ __forceinline__ f32x16 mma(f32x16 c, u32x4 a, u32x4 b) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ u32x4 operand(const f32x16& s, int i) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = __float_as_uint(s[i + j]);
    return r;
  }
  static __device__ __forceinline__ u32x4 only(u32x4 x, int j, bool here) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = here && k == j ? x[k] : 0u;
    return x;
  }
  static __device__ __forceinline__ uint32_t odd_bits(uint32_t x) { return (x & 0x7f800000u) + 0x00800000u; }
  static __device__ __forceinline__ u32x4 odd_part(u32x4 x) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (x[j] & 0x7f800000u) == 0x7f800000u ? x[j] : 0u;
    return r;
  }
  static __device__ __forceinline__ float dot(u32x4 x, u32x4 y) {
    float r = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) r = fmaf(__uint_as_float(x[j]), __uint_as_float(y[j]), r);
    return r;
  }
};

// Token (key or row) of accumulator register i, in its block of 32.
__device__ __forceinline__ int token_of(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// A tile of rows of D elements in LDS, kStride bytes apart: 32 more than a row, so that the 8 rows that 8 lanes read
// 16 bytes of lie in different banks (and the 4 rows of 64 bytes of a transposed read meet in few), and every
// address is a lane's own offset plus a constant.  (Rows without a gap, chunks exchanged by row: no conflict at all,
// but an instruction an address, a sixth of the loop's.)
template <bool BF, int D>
struct Tile {
  static constexpr int kRow = D * (BF ? 2 : 4), kStride = kRow + 32;
  static constexpr int kChunks = kRow / 16, kSteps = kChunks / 2, kBlocks = D / 32;

  int straight, across;  // byte offsets of this lane
  __device__ __forceinline__ Tile() {
    const int l = threadIdx.x & 63, h = l >> 5, a = l & 15;
    straight = (l & 31) * kStride + 16 * h;
    across = BF ? (4 * h + (a >> 2)) * kStride + 32 * ((l >> 4) & 1) + 8 * (a & 3) : 4 * h * kStride + 4 * (l & 31);
  }
  // Step s of the sum over a row's elements, rows row0 .. row0+31.
  __device__ __forceinline__ u32x4 rows(const char* base, int row0, int s) const {
    return *(const u32x4*)(base + straight + row0 * kStride + 32 * s);
  }
  // Elements 32 b .. 32 b + 31 of the tokens that an operand from kRegs accumulator registers on (from register
  // i of the block of 32 tokens at token0) stands for, transposed.
  __device__ __forceinline__ u32x4 columns(const char* base, int token0, int i, int b) const {
    const char* p = base + across + (token0 + 2 * i) * kStride;
    if constexpr (BF) {
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 64 * b));
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 64 * b + 8 * kStride));
      const u32x2 u = __builtin_bit_cast(u32x2, x), v = __builtin_bit_cast(u32x2, y);
      return u32x4{u[0], u[1], v[0], v[1]};
    } else {
      u32x4 r;
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = *(const uint32_t*)(p + j * kStride + 128 * b);
      return r;
    }
  }
};

// c += a b where a may hold infinities and NaN of tokens that a lane does not see: the others at once, so that their
// sum is what it is without these; then these token by token, and the lane takes token t (of the 32 that the
// registers from i on are part of) where lo <= t <= hi.
template <bool BF>
__device__ __forceinline__ void mma_seen(f32x16& c, u32x4 a, u32x4 b, int i, int lo, int hi) {
  const int half = (threadIdx.x >> 5) & 1;
  const u32x4 rest = Type<BF>::odd_part(a);
  c = Type<BF>::mma(c, a ^ rest, b);
#pragma unroll 1
  for (int j = 0; j < Type<BF>::kRegs; ++j) {
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      const u32x4 one = Type<BF>::only(rest, j, half == h);
      if (!__any(one[0] | one[1] | one[2] | one[3])) continue;
      const f32x16 p = Type<BF>::mma(f32x16{}, one, Type<BF>::only(b, j, half == h));
      const int t = token_of(i + j, h);
      const bool seen = t >= lo && t <= hi;
#pragma unroll
      for (int e = 0; e < 16; ++e) c[e] = seen ? c[e] + p[e] : c[e];
    }
  }
}

// Sequence whose tiles hold slot `slot`: the tiles (of 2^shift rows, per_token rows a token) of sequence i take
// slots first(i) .. , first(i) = rows before it / tile + i, which leaves room for every tile and at most one
// slot free.  Offsets are taken into [0, tokens], so that whatever they are nothing out of bounds is touched.
struct Place {
  int begin, end;  // tokens
  int sequence, tile;
};
__device__ __forceinline__ int offset_of(const int32_t* offsets, int i, int tokens) {
  return min(max(offsets[i], 0), tokens);
}
__device__ __forceinline__ Place find_place(const int32_t* offsets, int n, int tokens, int slot, int per_token, int shift) {
  const int lane = threadIdx.x & 63;
  const auto first = [&](int i) { return (int)(((int64_t)offset_of(offsets, i, tokens) * per_token >> shift) + i); };
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    const unsigned long long m = __ballot(i < n && first(lo + min(i, n - 1)) <= slot);
    const int j = m ? 63 - __builtin_clzll(m) : 0;
    lo += j * step;
    n = min(step, n - j * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  Place p;
  p.sequence = lo;
  p.begin = offset_of(offsets, lo, tokens);
  p.end = max(p.begin, offset_of(offsets, lo + 1, tokens));
  p.tile = slot - (int)(((int64_t)p.begin * per_token >> shift) + lo);
  return p;
}

// r / hpk by inv = ceil(2^32 / hpk) (at most one too large for r below 2^31).
__device__ __forceinline__ int divide_rows(int r, int hpk, uint32_t inv) {
  if (hpk == 1) return r;
  const int t = (int)__umulhi((uint32_t)r, inv);
  return t * hpk > r ? t - 1 : t;
}

// Rows of a tensor in registers between memory and LDS: `ROWS` of a tile, by `THREADS` threads.  from() sets the
// first tile's place, each load() goes on by a tile.
template <bool BF, int D, int ROWS, int THREADS>
struct Stage {
  using T = Tile<BF, D>;
  static constexpr int kPer = ROWS * T::kChunks / THREADS, kStep = THREADS / T::kChunks;
  static_assert(ROWS * T::kChunks % THREADS == 0 && THREADS % T::kChunks == 0, "whole chunks a thread");
  u32x4 x[kPer];
  const char* next;  // of the thread's first row
  static __device__ __forceinline__ int row(int i) { return (int)threadIdx.x / T::kChunks + i * kStep; }
  static __device__ __forceinline__ int chunk() { return (int)threadIdx.x % T::kChunks; }
  // Rows of tokens from `first` on, `stride` bytes apart.
  __device__ __forceinline__ void from(const char* base, int64_t stride, int first) {
    next = base + (first + row(0)) * stride + chunk() * 16;
  }
  // The tile of rows first ..; behind the last, row end - 1 again (end > first).
  __device__ __forceinline__ void load(int64_t stride, int first, int end) {
    if (first + ROWS <= end) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = *(const u32x4*)(next + i * kStep * stride);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = *(const u32x4*)(next + (min(first + row(i), end - 1) - first - row(0)) * stride);
    }
    next += ROWS * stride;
  }
  // Rows first .. of a group's heads, alike; `inv` as in divide_rows.
  __device__ __forceinline__ void load_rows(const char* base, int64_t stride, int64_t head, int first, int end, int hpk,
                                            uint32_t inv) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int r = min(first + row(i), end - 1), t = divide_rows(r, hpk, inv);
      x[i] = *(const u32x4*)(base + t * stride + (r - t * hpk) * head + chunk() * 16);
    }
  }
  __device__ __forceinline__ void store(char* lds) const {
    char* p = lds + row(0) * T::kStride + chunk() * 16;
#pragma unroll
    for (int i = 0; i < kPer; ++i) *(u32x4*)(p + i * kStep * T::kStride) = x[i];
  }
  __device__ __forceinline__ bool odd() const {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) r |= Type<BF>::odd_bits(x[i][j]);
    return r & (BF ? 0x80008000u : 0x80000000u);
  }
};

// Operands of a lane's own row (or key), straight from memory.
template <int STEPS>
__device__ __forceinline__ void load_operands(u32x4 (&f)[STEPS], const char* row, bool there) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    f[s] = u32x4{0, 0, 0, 0};
    if (there) f[s] = *(const u32x4*)(row + (2 * s + half) * 16);
  }
}

// Operands of a block of 32 rows, asked for ahead of the products that take them: what the compiler would move to
// their use, two at a time, each pair waiting for LDS.
template <int STEPS, class T>
__device__ __forceinline__ void fetch_rows(u32x4 (&f)[STEPS], const T& tile, const char* base, int row0) {
#pragma unroll
  for (int e = 0; e < STEPS; ++e) f[e] = tile.rows(base, row0, e);
  __builtin_amdgcn_sched_barrier(0);
}
// N times a matrix instruction, then an LDS load: the order of the code ahead of it.
template <int N>
__device__ __forceinline__ void paired() {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
}

// Elements 32 b .. 32 b + 31 of a lane's row of results times `by`: register i holds element token_of(i).
template <bool BF>
__device__ __forceinline__ void store_block(const f32x16& acc, float by, char* row, int b, bool there) {
  const int half = (threadIdx.x >> 5) & 1;
  if constexpr (BF) {
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = 4 * q + 2 * k;
        w[k] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)(acc[i] * by)) |
               (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)(acc[i + 1] * by)) << 16;
      }
      // two halves of 16 bytes each from two lanes: 8 elements from `half` on
      const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
      if (there) *(u32x4*)(row + 64 * b + 16 * q + 16 * half) = u32x4{x[0], y[0], x[1], y[1]};
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = acc[4 * q + k] * by;
      if (there) *(f32x4*)(row + 128 * b + 32 * q + 16 * half) = v;
    }
  }
}

// Sums over the S groups of a work-group's wavefronts, in group order, in the registers of group 0.  buffer: 4 KiB a
// wavefront.
template <int C, int S, int N>
__device__ __forceinline__ void join(f32x16 (&acc)[N], char* buffer) {
  if constexpr (S > 1) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int b = 0; b < N; ++b) {
      __syncthreads();
      if (wave >= C)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *(f32x4*)(buffer + ((wave * 4 + i / 4) * 64 + lane) * 16) = f32x4{acc[b][i], acc[b][i + 1], acc[b][i + 2], acc[b][i + 3]};
      __syncthreads();
      if (wave < C)
#pragma unroll
        for (int g = 1; g < S; ++g)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const f32x4 x = *(const f32x4*)(buffer + (((g * C + wave) * 4 + i / 4) * 64 + lane) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[b][i + j] += x[j];
          }
    }
  }
}

// ---- walks that several work-groups share ----
// One sequence's few rows over many keys (or a key over many rows) would be one long walk on one CU.  Work-groups of 32
// rows (C = 1) share it: each takes a run of its tiles, its results go to memory, and the last one to arrive adds
// them up in their order (nothing waits).  Measured, without and with (us): one token over 100000 keys 1358, 93; eight
// over 300 to 8000 keys 89, 46; the gradient of four fp32 sequences of 1 to 300 tokens 70, 38.  Work-groups of 64 rows
// have no registers left for it, and more than two a CU are slower (the chain of a small part is as long).
constexpr int kMostParts = 32;
template <bool BF>
constexpr int kLeastTiles = BF ? 2 : 1;  // a part; an fp32 tile takes as long as handing a part over

// The place of a work-group: walk `slot` of head g, and part `part` of the walk.  Parts that are not needed come last.
struct Walker {
  int g, slot, part, id;
  __device__ __forceinline__ Walker(const AttendShape& a, bool shared) {
    const int i = (int)(blockIdx.x / (unsigned)a.kv_heads);
    g = (int)blockIdx.x - i * a.kv_heads;
    part = shared ? (int)((unsigned)i / (unsigned)a.slots) : 0;
    slot = i - part * a.slots;
    id = slot * a.kv_heads + g;
  }
};
// Its tiles, first .. first + n - 1 of a walk of `tiles`, which takes `parts` of them; `part` may be none of these.
struct Share {
  int parts, first, n;
  __device__ __forceinline__ Share(int tiles, int part, int most, int least) {
    parts = min(most, max(1, tiles / least));
    first = (int)((int64_t)tiles * part / parts), n = (int)((int64_t)tiles * (part + 1) / parts) - first;
  }
};

__device__ __forceinline__ void publish(float* p, float x, float y) {  // past the caches of this XCD
  const uint64_t w = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
  __hip_atomic_store((uint64_t*)p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 collect(const float* p) {
  const uint64_t w = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return float2{__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32))};
}

// A block of results in a wavefront's place `at` of the parts' results: 1024 floats.
__device__ __forceinline__ void publish_block(float* at, const f32x16& x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 16; i += 2) publish(at + (i / 2 * 64 + lane) * 2, x[i], x[i + 1]);
}
// c = c * keep + the block * by
__device__ __forceinline__ void collect_block(f32x16& c, const float* at, float keep, float by) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const float2 x = collect(at + (i / 2 * 64 + lane) * 2);
    c[i] = fmaf(x.x, by, c[i] * keep), c[i + 1] = fmaf(x.y, by, c[i + 1] * keep);
  }
}

// Whether this work-group is the last of `parts` to come here, with what it published.  Leaves the counter 0.
__device__ __forceinline__ bool arrive(int32_t* counter, int parts) {
  __shared__ bool last;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);  // this thread's stores have reached the coherence point
  __syncthreads();
  if (threadIdx.x == 0) {
    last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
  }
  __syncthreads();
  return last;
}

// Sizes of a kernel of C columns and S splits: tokens of a tile, buffers of tiles, LDS.  `values`: bytes ahead.
template <bool BF, int D, int C, int S, int BLOCK>
struct Shape {
  static constexpr int kThreads = 64 * C * S;
  static constexpr int kBlock = BLOCK;  // tokens of a group's tile
  static constexpr int kTokens = kBlock * S;
  static constexpr int kBuffers = S == 1 ? 2 : 1;
  static constexpr int kTile = kTokens * Tile<BF, D>::kStride;
  static constexpr int kJoin = S > 1 ? C * S * 4096 : 0;
  static constexpr int kLds = 2 * kBuffers * kTile > kJoin ? 2 * kBuffers * kTile : kJoin;
};

// Walks tiles 0 .. n-1: load(t) brings the next tile's rows into registers, store(buffer, t) takes them into LDS,
// use(buffer, t) reads them there.  Two buffers: loads of a tile are in flight while the one before is used.
template <int BUFFERS, class Load, class Store, class Use>
__device__ __forceinline__ void walk(int n, Load load, Store store, Use use) {
  if (n <= 0) return;
  load(0);
  __syncthreads();
  store(0, 0);
  for (int t = 0; t < n; ++t) {
    __syncthreads();
    if (t + 1 < n) load(t + 1);
    __builtin_amdgcn_sched_barrier(0);
    use(BUFFERS == 2 ? t & 1 : 0, t);
    if (t + 1 < n) {
      if (BUFFERS == 1) __syncthreads();
      store(BUFFERS == 2 ? (t + 1) & 1 : 0, t + 1);
    }
  }
}

// The rows of a work-group and of its wavefronts, as the kernels of o and of dq have them.
template <int C>
struct Rows {
  Place p;
  int rows, row0, kb, keys, shift, token, head, last, seen_all, seen_any, seen_first, seen_last;
  int64_t q_token;
  bool there;
  // false: nothing to do
  __device__ __forceinline__ bool find(const AttendShape& a, const Walker& at) {
    constexpr int BM = 32 * C;
    const int g = at.g, slot = a.slots - 1 - at.slot;  // the longest rows first
    p = find_place(a.q_offsets, a.sequences, a.q_tokens, slot, a.hpk, __builtin_ctz(BM));
    rows = (p.end - p.begin) * a.hpk, row0 = p.tile * BM;
    if (p.tile < 0 || row0 >= rows) return false;
    kb = offset_of(a.k_offsets, p.sequence, a.k_tokens);
    keys = max(0, offset_of(a.k_offsets, p.sequence + 1, a.k_tokens) - kb);
    shift = keys - (p.end - p.begin);
    const int wrow = row0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % C * 32;
    const int row = min(wrow + ((int)threadIdx.x & 31), rows - 1);
    there = wrow + ((int)threadIdx.x & 31) < rows;
    token = divide_rows(row, a.hpk, a.hpk_inv), head = g * a.hpk + row - token * a.hpk;
    q_token = p.begin + token;
    last = there ? token + shift : -1;  // the last key that the row sees
    // .. that the wavefront's first, and its last row see, and the work-group's
    seen_all = wrow < rows ? divide_rows(wrow, a.hpk, a.hpk_inv) + shift : -1;
    seen_any = wrow < rows ? divide_rows(min(wrow + 31, rows - 1), a.hpk, a.hpk_inv) + shift : -1;
    seen_first = divide_rows(row0, a.hpk, a.hpk_inv) + shift;
    seen_last = divide_rows(min(row0 + BM, rows) - 1, a.hpk, a.hpk_inv) + shift;
    return true;
  }
};

// ---- o and lse -----------------------------------------------------------------
// Bound by the chain of a tile: first product, maximum, exponentials, second product, each of which waits for the one
// before, with two wavefronts a SIMD to fill in (256 registers each).  Four packed prompts of 256 to 4096 tokens, 32
// heads of 128 on 8 KV heads: 203 to 221 us (one card and another), 820 to 890 TFLOP/s, where a large matrix product of
// the same type reaches 1290.
// Leaving out loads, exponentials or either product gained a tenth each; wavefronts half a tile apart (three buffers),
// operands asked for a whole product ahead, and two work-groups of 128 rows a CU gained nothing.
template <bool BF, int D, int C, int S>
__global__ __launch_bounds__(64 * C * S, C * S >= 8 ? 2 : 1) void attend_kernel(const AttendArgs a) {
  constexpr bool kShared = C == 1;
  using T = Tile<BF, D>;
  using H = Shape<BF, D, C, S, (BF && C > 1) ? 64 : 32>;
  constexpr int BN = H::kBlock, NB = BN / 32, R = Type<BF>::kRegs;
  __shared__ __attribute__((aligned(16))) char lds[H::kLds];
  __shared__ float maxima[S][C * 32], sums[S][C * 32];
  __shared__ int odd;  // V holds an infinity or NaN in a tile that some rows do not see
  Rows<C> w;
  const Walker at(a, kShared);
  if (!w.find(a, at)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int column = wave % C, group = wave / C, g = at.g;
  const Share share(w.seen_last < 0 ? 0 : w.seen_last / H::kTokens + 1,
                    at.part, kShared ? a.parts : 1, kLeastTiles<BF>);
  if (at.part >= share.parts) return;
  // of the walk: [parts][blocks][1024], [parts][32][2]
  float* results = a.part + (int64_t)at.id * a.parts * (32 * (D + 2));
  float* statistics = results + a.parts * (32 * D);
  const char* kbase = a.k + w.kb * a.k_row + g * a.k_head;
  const char* vbase = a.v + w.kb * a.v_row + g * a.v_head;
  const float c = a.scale * kLog2e;
  const T tile;
  if (threadIdx.x == 0) odd = 0;

  // Joins the groups; blocks b0 .. of the result, to its rows or to the parts'.
  const auto finish = [&](auto& acc, float m, float sum, int b0, bool to_parts) {
    constexpr int KB = sizeof(acc) / sizeof(f32x16);
    if constexpr (S > 1) {
      __syncthreads();
      if (half == 0) maxima[group][column * 32 + lane] = m, sums[group][column * 32 + lane] = sum;
      __syncthreads();
      const int own = column * 32 + (lane & 31);
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < S; ++i) top = fmaxf(top, maxima[i][own]);
      const float base = top == -INFINITY ? 0.f : top;
      const float by = exp2_((m - base) * c);
#pragma unroll
      for (int b = 0; b < KB; ++b) acc[b] *= by;
      m = top, sum = 0.f;
#pragma unroll
      for (int i = 0; i < S; ++i) sum = fmaf(sums[i][own], exp2_((maxima[i][own] - base) * c), sum);
      join<C, S>(acc, lds);
      if (group > 0) return;
      if (kShared && to_parts) {
        if (half == 0) publish(statistics + (at.part * 32 + lane) * 2, m, sum);
#pragma unroll
        for (int b = 0; b < KB; ++b) publish_block(results + (at.part * T::kBlocks + b0 + b) * 1024, acc[b]);
        return;
      }
    }
    const float by = w.last < 0 ? 0.f : 1.f / sum;
#pragma unroll
    for (int b = 0; b < KB; ++b) store_block<BF>(acc[b], by, a.o + w.q_token * a.o_row + w.head * a.o_head, b0 + b, w.there);
    if (w.there && half == 0 && a.lse)
      a.lse[w.q_token * a.q_heads + w.head] =
          w.last < 0 ? -INFINITY : (m == -INFINITY ? 0.f : m * a.scale) + __log2f(sum) * kLn2;
  };
  const auto pass = [&](auto careful, int b0) {
    constexpr int KB = careful ? 1 : T::kBlocks;  // blocks of 32 elements of the result, from b0 on
    Stage<BF, D, H::kTokens, H::kThreads> sk, sv;
    sk.from(kbase, a.k_row, share.first * H::kTokens);
    sv.from(vbase, a.v_row, share.first * H::kTokens);
    u32x4 q[T::kSteps];
    load_operands(q, a.q + w.q_token * a.q_row + w.head * a.q_head, w.there);
    f32x16 acc[KB] = {};
    float m = -INFINITY, sum = 0.f;
    const float slack = kSlack / c;
    walk<careful ? 1 : H::kBuffers>(
        share.n,
        [&](int t) {
          sk.load(a.k_row, (share.first + t) * H::kTokens, w.keys);
          sv.load(a.v_row, (share.first + t) * H::kTokens, w.keys);
        },
        [&](int buffer, int t) {
          sk.store(lds + 2 * buffer * H::kTile);
          sv.store(lds + (2 * buffer + 1) * H::kTile);
          if (!careful && (share.first + t + 1) * H::kTokens - 1 > w.seen_first && sv.odd()) odd = 1;
        },
        [&](int buffer, int t) {
          const int key0 = (share.first + t) * H::kTokens + group * BN;
          if (key0 > w.seen_any) return;
          const char* lk = lds + 2 * buffer * H::kTile + group * BN * T::kStride;
          const char* lv = lk + H::kTile;
          f32x16 s[NB] = {};
          u32x4 f[T::kSteps];
          fetch_rows(f, tile, lk, 0);
#pragma unroll
          for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int e = 0; e < T::kSteps; ++e) {
              s[n] = Type<BF>::mma(s[n], f[e], q[e]);
              if (n + 1 < NB) f[e] = tile.rows(lk, 32 * n + 32, e);
            }
            if (n + 1 < NB) paired<T::kSteps>();
          }
          if (key0 + BN - 1 > w.seen_all) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int i = 0; i < 16; ++i) s[n][i] = key0 + 32 * n + token_of(i, half) <= w.last ? s[n][i] : -INFINITY;
          }
          float top = -INFINITY;
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
          top = fmaxf(top, other_half(top));
          // the sums keep their base until a score is 2^kSlack times it: fp32 has room, and the operands of the second
          // product are as exact at any size
          const bool grows = top > m + slack;
          if (__any(grows)) {
            const float by = grows ? exp2_((m - top) * c) : 1.f;  // (a row of its own: none goes by another's scores)
            sum *= by;
#pragma unroll
            for (int b = 0; b < KB; ++b) acc[b] *= by;
            m = grows ? top : m;
          }
          float off = m == -INFINITY ? 0.f : -m * c;
          if (__any(fabsf(off) > kFar)) {
            const float by = fabsf(off) > kFar ? m : 0.f;  // (again a row of its own)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int i = 0; i < 16; ++i) s[n][i] -= by;
            off = fabsf(off) > kFar ? 0.f : off;
          }
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              s[n][i] = exp2_(fmaf(s[n][i], c, off));
              sum += s[n][i];
            }
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += R) {
              const u32x4 p = Type<BF>::operand(s[n], i);
#pragma unroll
              for (int b = 0; b < KB; ++b) {
                const u32x4 v = tile.columns(lv, 32 * n, i, b0 + b);
                if constexpr (careful)
                  mma_seen<BF>(acc[b], v, p, i, 0, w.last - key0 - 32 * n);
                else
                  acc[b] = Type<BF>::mma(acc[b], v, p);
              }
            }
        });
    sum += other_half(sum);
    finish(acc, m, sum, b0, share.parts > 1);
  };
  pass(std::false_type{}, 0);
  __syncthreads();
  if (odd)
    for (int b = 0; b < T::kBlocks; ++b) {
      __syncthreads();
      pass(std::true_type{}, b);
    }
  if constexpr (kShared) {
    if (share.parts == 1 || !arrive(a.arrived + at.id, share.parts)) return;
    // the parts, in turn over the groups
    f32x16 acc[T::kBlocks] = {};
    float m = -INFINITY, sum = 0.f;
    for (int i = group; i < share.parts; i += S) {
      const float2 x = collect(statistics + (i * 32 + (lane & 31)) * 2);
      const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.f : top;
      const float keep = exp2_((m - base) * c), by = exp2_((x.x - base) * c);
      m = top, sum = fmaf(x.y, by, sum * keep);
#pragma unroll
      for (int b = 0; b < T::kBlocks; ++b) collect_block(acc[b], results + (i * T::kBlocks + b) * 1024, keep, by);
    }
    finish(acc, m, sum, 0, false);
  }
}

// -lse in powers of 2.  Where its roundings (lse's own, the product's, that of the scale) may come to powers that leave
// fp32, lower by twice their bound, so that no p is above 1.
__device__ __forceinline__ float base_of(float lse) {
  const float off = -lse * kLog2e, size = fminf(fabsf(off), 3e38f);
  return size > 0x1p26f ? off - size * 0x1p-21f : off;
}

// ---- dq (and D) ----------------------------------------------------------------
// The walk of the forward kernel with the scores' exponentials from lse: s^T and (v up)^T of a tile, ds^T from
// them, dq^T += K^T ds^T.  D = up.o of every row is left in a.delta for the kernel of dk and dv.
// Three products and no maximum: 158 us for eight sequences of 640 to 2560 tokens, 16 heads of 128 on 8 KV heads.
template <bool BF, int D, int C, int S>
__global__ __launch_bounds__(64 * C * S, C * S >= 8 ? 2 : 1) void attend_dq_kernel(const AttendGradArgs a) {
  constexpr bool kShared = C == 1;
  using T = Tile<BF, D>;
  using H = Shape<BF, D, C, S, (BF && (C > 2 || (C > 1 && D == 64))) ? 64 : 32>;
  constexpr int BN = H::kBlock, NB = BN / 32, R = Type<BF>::kRegs;
  __shared__ __attribute__((aligned(16))) char lds[H::kLds];
  __shared__ int odd;  // K holds an infinity or NaN in a tile that some rows do not see
  Rows<C> w;
  const Walker at(a, kShared);
  if (!w.find(a, at)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int group = wave / C, g = at.g;
  const Share share(w.seen_last < 0 ? 0 : w.seen_last / H::kTokens + 1,
                    at.part, kShared ? a.parts : 1, kLeastTiles<BF>);
  if (at.part >= share.parts) return;
  float* results = a.part + (int64_t)at.id * a.parts * (32 * D);  // of the walk: [parts][blocks][1024]
  const char* kbase = a.k + w.kb * a.k_row + g * a.k_head;
  const char* vbase = a.v + w.kb * a.v_row + g * a.v_head;
  const int64_t row = w.q_token * a.q_heads + w.head;
  const float c = a.scale * kLog2e, off = w.there ? base_of(a.lse[row]) : 0.f;
  const T tile;
  if (threadIdx.x == 0) odd = 0;

  const auto finish = [&](auto& acc, int b0, bool to_parts) {
    constexpr int KB = sizeof(acc) / sizeof(f32x16);
    join<C, S>(acc, lds);
    if (group > 0) return;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if (kShared && to_parts)
        publish_block(results + (at.part * T::kBlocks + b0 + b) * 1024, acc[b]);
      else
        store_block<BF>(acc[b], a.scale, a.dq + w.q_token * a.dq_row + w.head * a.dq_head, b0 + b, w.there);
    }
  };
  const auto pass = [&](auto careful, int b0) {
    constexpr int KB = careful ? 1 : T::kBlocks;
    Stage<BF, D, H::kTokens, H::kThreads> sk, sv;
    sk.from(kbase, a.k_row, share.first * H::kTokens);
    sv.from(vbase, a.v_row, share.first * H::kTokens);
    u32x4 q[T::kSteps], up[T::kSteps];
    float delta = 0.f;
    load_operands(q, a.o + w.q_token * a.o_row + w.head * a.o_head, w.there);
    load_operands(up, a.d_o + w.q_token * a.do_row + w.head * a.do_head, w.there);
#pragma unroll
    for (int s = 0; s < T::kSteps; ++s) delta += Type<BF>::dot(q[s], up[s]);
    delta += other_half(delta);
    load_operands(q, a.q + w.q_token * a.q_row + w.head * a.q_head, w.there);
    if (w.there && half == 0 && group == 0 && at.part == 0) a.delta[row] = delta;
    f32x16 acc[KB] = {};
    walk<careful ? 1 : H::kBuffers>(
        share.n,
        [&](int t) {
          sk.load(a.k_row, (share.first + t) * H::kTokens, w.keys);
          sv.load(a.v_row, (share.first + t) * H::kTokens, w.keys);
        },
        [&](int buffer, int t) {
          sk.store(lds + 2 * buffer * H::kTile);
          sv.store(lds + (2 * buffer + 1) * H::kTile);
          if (!careful && (share.first + t + 1) * H::kTokens - 1 > w.seen_first && sk.odd()) odd = 1;
        },
        [&](int buffer, int t) {
          const int key0 = (share.first + t) * H::kTokens + group * BN;
          if (key0 > w.seen_any) return;
          const char* lk = lds + 2 * buffer * H::kTile + group * BN * T::kStride;
          const char* lv = lk + H::kTile;
          const bool masked = key0 + BN - 1 > w.seen_all;
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            f32x16 s = {}, ds = {};
#pragma unroll
            for (int e = 0; e < T::kSteps; ++e) {
              s = Type<BF>::mma(s, tile.rows(lk, 32 * n, e), q[e]);
              ds = Type<BF>::mma(ds, tile.rows(lv, 32 * n, e), up[e]);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[i] = exp2_(fmaf(s[i], c, off)) * (ds[i] - delta);
            if (masked) {
#pragma unroll
              for (int i = 0; i < 16; ++i) ds[i] = key0 + 32 * n + token_of(i, half) <= w.last ? ds[i] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 16; i += R) {
              const u32x4 p = Type<BF>::operand(ds, i);
#pragma unroll
              for (int b = 0; b < KB; ++b) {
                const u32x4 k = tile.columns(lk, 32 * n, i, b0 + b);
                if constexpr (careful)
                  mma_seen<BF>(acc[b], k, p, i, 0, w.last - key0 - 32 * n);
                else
                  acc[b] = Type<BF>::mma(acc[b], k, p);
              }
            }
          }
        });
    finish(acc, b0, share.parts > 1);
  };
  pass(std::false_type{}, 0);
  __syncthreads();
  if (odd)
    for (int b = 0; b < T::kBlocks; ++b) {
      __syncthreads();
      pass(std::true_type{}, b);
    }
  if constexpr (kShared) {
    if (share.parts == 1 || !arrive(a.arrived + at.id, share.parts)) return;
    f32x16 acc[T::kBlocks] = {};
    for (int i = group; i < share.parts; i += S)
#pragma unroll
      for (int b = 0; b < T::kBlocks; ++b) collect_block(acc[b], results + (i * T::kBlocks + b) * 1024, 1.f, 1.f);
    finish(acc, 0, false);
  }
}

// ---- dk and dv -----------------------------------------------------------------
// A wavefront's 32 keys are the columns: s = Q k^T and up v^T over a tile of rows, p and ds from them, then
// dv^T += up^T p and dk^T += Q^T ds with the rows as the tokens of the sum.  A key is seen by the rows from
// (key - shift) hpk on.
//
// Registers: two operands and two results of 32 keys, 192 of them for bf16 heads of 128 and twice as many operands in
// fp32.  For bf16 the values' operand stays in LDS (a quarter more to read there; in registers the kernel spilled);
// fp32 heads of 128, and splits, take a wavefront's whole file.  bf16 keys of two wavefronts and four splits still spill, 15
// registers for heads of 128 and 12 for 64.
// Bound by LDS: of 32 x 32 products whose operands both serve once, 400 cycles of reads for 1024 of the matrix unit,
// and eight wavefronts on one LDS.  287 us for the sequences above (four products); work-groups of 256 keys, one a CU
// instead of two of 128, took 310.
template <bool BF, int D, int C, int S>
struct KeyShape {
  static constexpr int kThreads = 64 * C * S;
  static constexpr int kBlock = BF && D == 64 && C > 1 ? 64 : 32;  // rows of a group's tile
  static constexpr int kTokens = kBlock * S;
  static constexpr int kBuffers = S == 1 ? 2 : 1;
  static constexpr int kTile = kTokens * Tile<BF, D>::kStride;
  static constexpr bool kValues = D == 128 && (BF ? S == 1 || C * S == 8 : S > 1);  // in LDS
  static constexpr int kValueBytes = kValues ? 32 * C * Tile<BF, D>::kStride : 0;
  static constexpr int kJoin = S > 1 ? C * S * 4096 : 0;
  static constexpr int kTiles = 2 * kBuffers * kTile > kJoin ? 2 * kBuffers * kTile : kJoin;
};

template <bool BF, int D, int C, int S>
__global__ __launch_bounds__(64 * C * S, C * S >= 8 || (BF && S == 1) ? 2 : 1) void attend_dkv_kernel(const AttendGradArgs a) {
  constexpr bool kShared = C == 1;
  using T = Tile<BF, D>;
  using H = KeyShape<BF, D, C, S>;
  constexpr int BK = 32 * C, BR = H::kBlock, R = Type<BF>::kRegs;
  __shared__ __attribute__((aligned(16))) char lds[H::kTiles + H::kValueBytes];  // Q and d_o of tiles, V
  __shared__ __attribute__((aligned(16))) float stats[2][2][H::kTokens];         // -lse log2(e) and D of their rows
  __shared__ int odd;  // Q or d_o holds an infinity or NaN in a tile of which some keys are not seen, or behind its rows
  const Walker at(a, kShared);
  const int g = at.g, slot = at.slot;
  const Place p = find_place(a.k_offsets, a.sequences, a.k_tokens, slot, 1, __builtin_ctz(BK));
  const int keys = p.end - p.begin, key0 = p.tile * BK;
  if (p.tile < 0 || key0 >= keys) return;
  const int qb = offset_of(a.q_offsets, p.sequence, a.q_tokens);
  const int queries = max(0, offset_of(a.q_offsets, p.sequence + 1, a.q_tokens) - qb);
  const int shift = keys - queries, rows = queries * a.hpk;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int group = wave / C, wkey = key0 + wave % C * 32, key = wkey + (lane & 31);
  const bool there = key < keys;
  const auto first_row = [&](int k) { return max(0, k - shift) * a.hpk; };
  const int first = there ? first_row(key) : INT32_MAX;          // the first row that sees the key
  const int wfirst = wkey < keys ? first_row(wkey) : INT32_MAX;  // .. any, and all, of the wavefront's
  const int wall = first_row(min(wkey + 31, keys - 1));
  const int all = first_row(min(key0 + BK, keys) - 1);           // .. all of the work-group's
  const int from = first_row(key0);
  const Share share(rows > from ? (rows - from + H::kTokens - 1) / H::kTokens : 0,
                    at.part, kShared ? a.parts : 1, kLeastTiles<BF>);
  if (at.part >= share.parts) return;
  const int begin = from + share.first * H::kTokens;
  float* results = a.part + (int64_t)at.id * a.parts * (2 * 32 * D);  // of the walk: [parts][blocks][2][1024]
  const int64_t k_token = p.begin + (there ? key : key0);
  const char* qbase = a.q + qb * a.q_row + (int64_t)g * a.hpk * a.q_head;
  const char* dobase = a.d_o + qb * a.do_row + (int64_t)g * a.hpk * a.do_head;
  const float c = a.scale * kLog2e;
  const T tile;
  if (threadIdx.x == 0) odd = 0;
  char* values = lds + H::kTiles;
  if constexpr (H::kValues) {
    Stage<BF, D, BK, H::kThreads> sv;
    sv.from(a.v + p.begin * a.v_row + g * a.v_head, a.v_row, key0);
    sv.load(a.v_row, key0, keys);
    sv.store(values);
  }
  const char* own_values = values + wave % C * 32 * T::kStride;

  const auto finish = [&](auto& dk, auto& dv, int b0, bool to_parts) {
    constexpr int KB = sizeof(dk) / sizeof(f32x16);
    join<C, S>(dk, lds);
    join<C, S>(dv, lds);
    if (group > 0) return;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if (kShared && to_parts) {
        float* to = results + (at.part * T::kBlocks + b0 + b) * 2048;
        publish_block(to, dk[b]);
        publish_block(to + 1024, dv[b]);
      } else {
        store_block<BF>(dk[b], a.scale, a.dk + k_token * a.dk_row + g * a.dk_head, b0 + b, there);
        store_block<BF>(dv[b], 1.f, a.dv + k_token * a.dv_row + g * a.dv_head, b0 + b, there);
      }
    }
  };
  const auto pass = [&](auto careful, int b0) {
    constexpr int KB = careful ? 1 : T::kBlocks;
    Stage<BF, D, H::kTokens, H::kThreads> sq, so;
    u32x4 k[T::kSteps], v[H::kValues ? 1 : T::kSteps];
    load_operands(k, a.k + k_token * a.k_row + g * a.k_head, there);
    if constexpr (!H::kValues) load_operands(v, a.v + k_token * a.v_row + g * a.v_head, there);
    const float* stat = half ? a.delta : a.lse;
    float st = 0.f;  // the first wavefronts: one of a row's two values a lane
    f32x16 dk[KB] = {}, dv[KB] = {};
    walk<careful ? 1 : H::kBuffers>(
        share.n,
        [&](int t) {
          const int row0 = begin + t * H::kTokens, r = row0 + wave * 32 + (lane & 31);
          sq.load_rows(qbase, a.q_row, a.q_head, row0, rows, a.hpk, a.hpk_inv);
          so.load_rows(dobase, a.do_row, a.do_head, row0, rows, a.hpk, a.hpk_inv);
          st = 0.f;
          if (wave < H::kTokens / 32 && r < rows) {
            const int i = divide_rows(r, a.hpk, a.hpk_inv);
            st = stat[(int64_t)(qb + i) * a.q_heads + g * a.hpk + r - i * a.hpk];
          }
        },
        [&](int buffer, int t) {
          sq.store(lds + 2 * buffer * H::kTile);
          so.store(lds + (2 * buffer + 1) * H::kTile);
          if (wave < H::kTokens / 32) stats[buffer][half][wave * 32 + (lane & 31)] = half ? st : base_of(st);
          const int row0 = begin + t * H::kTokens;
          if (!careful && (row0 < all || row0 + H::kTokens > rows) && (sq.odd() || so.odd())) odd = 1;
        },
        [&](int buffer, int t) {
          const int row0 = begin + t * H::kTokens + group * BR;
          if (row0 + BR <= wfirst || row0 >= rows) return;
          const char* lq = lds + 2 * buffer * H::kTile + group * BR * T::kStride;
          const char* lo = lq + H::kTile;
          const bool masked = row0 < wall || row0 + BR > rows;
#pragma unroll
          for (int n = 0; n < BR; n += 32) {
            f32x16 s = {}, ds = {};
#pragma unroll
            for (int e = 0; e < T::kSteps; ++e) {
              s = Type<BF>::mma(s, tile.rows(lq, n, e), k[e]);
              ds = Type<BF>::mma(ds, tile.rows(lo, n, e), H::kValues ? tile.rows(own_values, 0, e) : v[H::kValues ? 0 : e]);
            }
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const f32x4 off = *(const f32x4*)&stats[buffer][0][group * BR + n + token_of(i, half)];
              const f32x4 delta = *(const f32x4*)&stats[buffer][1][group * BR + n + token_of(i, half)];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                s[i + j] = exp2_(fmaf(s[i + j], c, off[j]));
                ds[i + j] = s[i + j] * (ds[i + j] - delta[j]);
              }
            }
            if (masked) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int r = row0 + n + token_of(i, half);
                const bool seen = r >= first && r < rows;
                s[i] = seen ? s[i] : 0.f;
                ds[i] = seen ? ds[i] : 0.f;
              }
            }
#pragma unroll
            for (int i = 0; i < 16; i += R) {
              const u32x4 pw = Type<BF>::operand(s, i), dw = Type<BF>::operand(ds, i);
#pragma unroll
              for (int b = 0; b < KB; ++b) {
                const u32x4 o = tile.columns(lo, n, i, b0 + b), q = tile.columns(lq, n, i, b0 + b);
                if constexpr (careful) {
                  const int from = first - row0 - n, to = rows - 1 - row0 - n;  // rows of the block that see the key
                  mma_seen<BF>(dv[b], o, pw, i, from, to);
                  mma_seen<BF>(dk[b], q, dw, i, from, to);
                } else {
                  dv[b] = Type<BF>::mma(dv[b], o, pw);
                  dk[b] = Type<BF>::mma(dk[b], q, dw);
                }
              }
            }
          }
        });
    finish(dk, dv, b0, share.parts > 1);
  };
  pass(std::false_type{}, 0);
  __syncthreads();
  if (odd)
    for (int b = 0; b < T::kBlocks; ++b) {
      __syncthreads();
      pass(std::true_type{}, b);
    }
  if constexpr (kShared) {
    if (share.parts == 1 || !arrive(a.arrived + at.id, share.parts)) return;
    f32x16 dk[T::kBlocks] = {}, dv[T::kBlocks] = {};
    for (int i = group; i < share.parts; i += S)
#pragma unroll
      for (int b = 0; b < T::kBlocks; ++b) {
        const float* from = results + (i * T::kBlocks + b) * 2048;
        collect_block(dk[b], from, 1.f, 1.f);
        collect_block(dv[b], from + 1024, 1.f, 1.f);
      }
    finish(dk, dv, 0, false);
  }
}

// Slots of the tiles of `tile` rows (per_token rows a token).
int slots_of(int64_t tokens, int per_token, int sequences, int tile) { return (int)(tokens * per_token / tile + sequences); }

// Whether rows make `groups` work-groups of `tile` rows.  More rows a work-group are fewer bytes through LDS for each,
// fewer rows are more work-groups, with more splits each, for long walks over keys and for causal ones, which end at
// different times.  Measured (us; work-groups of 32, 64 and 256 rows; sequences x tokens, 16 heads of 128 on 8 KV heads):
//   bf16 o    4 x 256: 22 12 13    1 x 2048: 76 45 61    4 x 1024: 111 60 36    64 x 128: 152 73 37
//   bf16 dq   4 x 256: 22 16 19    1 x 2048: 90 55 83    4 x 1024: 122 75 54    64 x 128: 140 87 60
//   fp32 o    4 x 256: 38 29 65    1 x 2048: 228 190 505    4 x 1024: 269 205 259    4 x 4096: 3376 2756 2273
// so bf16 takes 64 and 256 rows as soon as they fill the GPU once.  fp32 products take eight times as long and are
// never waited for, so a GPU that is filled evenly to the end is worth more: 4 work-groups of 256 a CU, and of 64 two
// where walks are long (1 x 1024: 68 89; 300 to 800 tokens, 8 heads on 2: 57 73), one where they are short (20 sequences of
// 1 to 381 tokens: 69 55).
// dk and dv (32, 64 and 128 keys):
//   bf16      4 x 512: 47 33 57    4 x 1024: 119 93 113    8 x 2048: 757 493 461    64 x 128: 99 62 53
//   fp32      4 x 512: 147 151 292    4 x 1024: 391 465 571    4 x 2048: 1417 1272 1814    64 x 128: 208 176 325
constexpr int kCus = 256, kShortWalk = 384;  // kShortWalk: keys of a sequence, on average
bool fills(int64_t tokens, int per_token, int kv_heads, int tile, int groups) {
  return tokens * per_token / tile * kv_heads >= groups;
}

bool short_walks(const AttendShape& a) { return a.k_tokens / a.sequences <= kShortWalk; }

// Work-groups that may share a walk: as many as there is room for (two a CU), and as the longest walk there can be has
// tiles for.
void share_walks(AttendShape& a, bool shared, int64_t longest, int tile, int least) {
  const int64_t walks = (int64_t)a.slots * a.kv_heads, most = (longest + tile - 1) / tile / least;
  a.parts = shared ? (int)std::max<int64_t>(1, std::min({kAttendParts / walks, most, (int64_t)kMostParts})) : 1;
}

template <bool BF, int D, int C, int S>
hipError_t attend(AttendArgs& a, hipStream_t stream) {
  a.slots = slots_of(a.q_tokens, a.hpk, a.sequences, C * 32);
  share_walks(a, C == 1, a.k_tokens, 32 * S, kLeastTiles<BF>);
  const dim3 grid((unsigned)a.slots * a.kv_heads * a.parts), block(64 * C * S);
  hipLaunchKernelGGL((attend_kernel<BF, D, C, S>), grid, block, 0, stream, a);
  return hipGetLastError();
}
template <bool BF, int D, int C, int S>
hipError_t attend_dq(AttendGradArgs& a, hipStream_t stream) {
  a.slots = slots_of(a.q_tokens, a.hpk, a.sequences, C * 32);
  share_walks(a, C == 1, a.k_tokens, 32 * S, kLeastTiles<BF>);
  const dim3 grid((unsigned)a.slots * a.kv_heads * a.parts), block(64 * C * S);
  hipLaunchKernelGGL((attend_dq_kernel<BF, D, C, S>), grid, block, 0, stream, a);
  return hipGetLastError();
}
template <bool BF, int D, int C, int S>
hipError_t attend_dkv(AttendGradArgs& a, hipStream_t stream) {
  a.slots = slots_of(a.k_tokens, 1, a.sequences, C * 32);
  share_walks(a, C == 1, (int64_t)a.q_tokens * a.hpk, 32 * S, kLeastTiles<BF>);
  const dim3 grid((unsigned)a.slots * a.kv_heads * a.parts), block(64 * C * S);
  hipLaunchKernelGGL((attend_dkv_kernel<BF, D, C, S>), grid, block, 0, stream, a);
  return hipGetLastError();
}

template <bool BF, int D>
hipError_t attend(AttendArgs& a, hipStream_t stream) {
  constexpr bool kLarge = !BF && D == 128;  // rows of 512 bytes
  if (fills(a.q_tokens, a.hpk, a.kv_heads, 256, kCus * (BF ? 1 : 4))) return attend<BF, D, 8, 1>(a, stream);
  if (fills(a.q_tokens, a.hpk, a.kv_heads, 64, kCus * (BF || short_walks(a) ? 1 : 2)))
    return attend<BF, D, 2, kLarge ? 2 : 4>(a, stream);
  return attend<BF, D, 1, kLarge ? 4 : 8>(a, stream);
}

template <bool BF, int D>
hipError_t attend_dq(AttendGradArgs& a, hipStream_t stream) {
  constexpr bool kLarge = !BF && D == 128;
  if (fills(a.q_tokens, a.hpk, a.kv_heads, 256, kCus * (BF ? 1 : 4))) return attend_dq<BF, D, 8, 1>(a, stream);
  if (fills(a.q_tokens, a.hpk, a.kv_heads, 64, kCus * (BF || short_walks(a) ? 1 : 2)))
    return attend_dq<BF, D, 2, kLarge ? 2 : 4>(a, stream);
  return attend_dq<BF, D, 1, D == 128 ? 4 : 8>(a, stream);
}

template <bool BF, int D>
hipError_t attend_grad(AttendGradArgs& a, hipStream_t stream) {
  const hipError_t e = attend_dq<BF, D>(a, stream);
  if (e != hipSuccess) return e;
  if constexpr (BF)
    if (fills(a.k_tokens, 1, a.kv_heads, 128, kCus * 2)) return attend_dkv<BF, D, 4, 1>(a, stream);
  if (fills(a.k_tokens, 1, a.kv_heads, 64, kCus * (BF ? 1 : 4)))
    return attend_dkv<BF, D, 2, !BF && D == 128 ? 2 : 4>(a, stream);
  return attend_dkv<BF, D, 1, BF && D == 64 ? 8 : 4>(a, stream);
}

}  // namespace

hipError_t launch_attend(AttendArgs& a, bool bf16, int head_dim, hipStream_t stream) {
  return head_dim == 64 ? (bf16 ? attend<true, 64>(a, stream) : attend<false, 64>(a, stream))
                        : (bf16 ? attend<true, 128>(a, stream) : attend<false, 128>(a, stream));
}

hipError_t launch_attend_grad(AttendGradArgs& a, bool bf16, int head_dim, hipStream_t stream) {
  return head_dim == 64 ? (bf16 ? attend_grad<true, 64>(a, stream) : attend_grad<false, 64>(a, stream))
                        : (bf16 ? attend_grad<true, 128>(a, stream) : attend_grad<false, 128>(a, stream));
}

}  // namespace infs
