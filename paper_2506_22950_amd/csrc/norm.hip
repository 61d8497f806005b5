// Norms of heads with the rotation in the same pass, and their gradient.
//
// For a head x of d elements, weights w, n = sqrt(sum x^2 / d + eps):
//   z = w x / n,   out = R z       (R: the rotation of rotary.hip, amplitude included)
// and with g = R^T d_out, the rotation by the negative angle:
//   d_x = (w g - x (sum w g x) / (d n^2)) / n,   d_w = sum over tokens and heads of g x / n
// Everything between a load and a store is fp32, rounded once.
//
// Bound by memory (the gradient too: it reads x and d_out, writes d_x).  A group of lanes, a power of two, holds
// a head in registers, so that its sums take a few exchanges inside a wavefront and nothing is read twice.
// 7424 tokens, 40 heads of 128 in bf16: 34.7 us, 4.4 TB/s (a large copy: 5.2).  16 slots, 24 heads: 4.8 us, a
// launch's ends and one chain of loads, sums and stores.
// Angles, and the weights in fp32, are put into LDS once per work-group and token.
#include "ops.h"
#include "rows.h"

#include <algorithm>

namespace infs {
namespace {

// What a lane holds of a head.
enum Unit {
  kElement,  // elements l, l + 64, ..: any sizes and alignment, a wavefront a head
  kChunk,    // 16 bytes, of heads of whole, aligned chunks; halves: partners come through LDS
  kPairs     // halves: 16 bytes of first and 16 bytes of second elements (a chunk behind the rotated part),
             // where the pairs too are whole chunks
};

template <bool BF, bool IL, int UNIT>
struct Head {
  using E = Elem<BF>;
  static constexpr int N = UNIT == kElement ? 1 : E::N, ES = BF ? 2 : 4;
  static constexpr int M = UNIT == kElement ? 4 : UNIT == kPairs ? 2 * N : N;  // elements of a lane
  static constexpr bool kExchange = UNIT == kElement || (UNIT == kChunk && !IL);
  // kChunk: angles of a chunk are apart in the table, so that those of lanes next to each other lie together
  static constexpr int kApart = UNIT != kChunk ? 1 : IL ? N / 2 : N;
  static constexpr int kTable = UNIT == kChunk ? kRotaryTable * N : kRotaryTable;
  static constexpr int kExchangeFloats = UNIT == kElement ? INFS_ROTARY_MAX_DIM / 64 : N;  // a thread

  int head_dim, pairs, u, columns;
  __device__ __forceinline__ Head(const RotaryArgs& a, int lane) {
    head_dim = a.head_dim, pairs = a.pairs, u = lane;
    columns = (pairs + kApart - 1) / kApart;
  }
  __device__ __forceinline__ int place_of(int t, int f) const { return (t * kApart + f % kApart) * columns + f / kApart; }
  __device__ __forceinline__ bool turned() const { return u < pairs / N; }  // kPairs
  // Element of the head that value m is, and whether there is one.
  __device__ __forceinline__ int element(int m) const {
    if (UNIT == kElement) return u + 64 * m;
    if (UNIT == kChunk) return u * N + m;
    return turned() ? (m < N ? u * N + m : pairs + u * N + m - N) : 2 * pairs + (u - pairs / N) * N + m;
  }
  __device__ __forceinline__ bool has(int m) const {
    if (UNIT == kPairs && m >= N) return turned();
    return element(m) < head_dim;
  }
  __device__ __forceinline__ void load(const char* p, bool there, float (&x)[M]) const {
    if constexpr (UNIT == kElement) {
#pragma unroll
      for (int m = 0; m < M; ++m) x[m] = there && has(m) ? E::load(p, element(m)) : 0.f;
    } else {
#pragma unroll
      for (int m = 0; m < M; m += N) {
        u32x4 v = {0, 0, 0, 0};
        if (there && has(m)) v = *(const u32x4*)(p + element(m) * ES);
#pragma unroll
        for (int j = 0; j < N; ++j) x[m + j] = E::get(v, j);
      }
    }
  }
  __device__ __forceinline__ void store(char* p, bool there, const float (&x)[M]) const {
    if constexpr (UNIT == kElement) {
#pragma unroll
      for (int m = 0; m < M; ++m)
        if (there && has(m)) E::store(p, element(m), x[m]);
    } else {
#pragma unroll
      for (int m = 0; m < M; m += N) {
        float y[N];
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = x[m + j];
        if (there && has(m)) __builtin_nontemporal_store(E::pack(y), (u32x4*)(p + element(m) * ES));
      }
    }
  }
  // y = the rotation of x by the angles of one token, or (BACK) its transpose.  exchange: the head's floats in LDS.
  template <bool BACK>
  __device__ __forceinline__ void rotate(const float2* cs, float* exchange, const float (&x)[M], float (&y)[M]) const {
    if constexpr (UNIT == kPairs) {
      cs += turned() ? u * N : 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float2 w = cs[turned() ? j : 0];
        const float s = BACK ? -w.y : w.y;
        y[j] = turned() ? fmaf(x[j], w.x, -(x[N + j] * s)) : x[j];
        y[N + j] = fmaf(x[N + j], w.x, x[j] * s);
      }
    } else {
      if constexpr (kExchange) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last head's reads are done
#pragma unroll
        for (int m = 0; m < M; ++m)
          if (has(m)) exchange[element(m)] = x[m];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int e = has(m) ? element(m) : 0;
        const bool rest = e >= 2 * pairs, second = IL ? e & 1 : e >= pairs;
        const int pair = rest ? 0 : IL ? e >> 1 : second ? e - pairs : e;
        float other;
        if constexpr (!kExchange)
          other = x[m ^ 1];
        else
          other = exchange[rest ? e : IL ? e ^ 1 : second ? e - pairs : e + pairs];
        const float2 w = cs[place_of(0, pair)];
        const float s = BACK ? -w.y : w.y;
        y[m] = rest ? x[m] : fmaf(x[m], w.x, second ? other * s : -(other * s));
      }
    }
  }
};

// Sum over a group of lanes (a power of two), the same in all of them.
__device__ __forceinline__ float group_sum(float x, int group) {
  for (int i = 1; i < group; i <<= 1) x += __shfl_xor(x, i);
  return x;
}

// Sum of squares of a lane's elements.
template <int M>
__device__ __forceinline__ float squares_of(const float (&x)[M]) {
  float s = 0.f;
#pragma unroll
  for (int m = 0; m < M; ++m) s = fmaf(x[m], x[m], s);
  return s;
}

// n^2 = mean square + eps of a head, where it is outside (2^-90, 2^126) (rare): there squares may have left fp32's range, or
// lost what n^2 is made of.  The head is then taken times f = 2^-70 or 2^96, and eps times f^2, which brings any n^2 but 0 and
// infinity to 2^-114 .. 2^116 and is exact but for elements that become denormal (2^-119 of n and less); n is f times what it
// was.  The wavefront takes the branch as one.  Without and with it (us): 7424 tokens, 40 heads of 128 in bf16 34.8, 34.9; the
// gradient of 8192 tokens, 24 heads 43.5, 43.8.
__device__ __forceinline__ bool out_of_range(float n2) { return !(n2 > 0x1p-90f && n2 < 0x1p126f); }
template <int M>
__device__ __forceinline__ float scale_heads(float (&x)[M], float& n2, const NormWeights& n) {
  const float f = !out_of_range(n2) ? 1.f : n2 < 1.f ? 0x1p96f : 0x1p-70f;
#pragma unroll
  for (int m = 0; m < M; ++m) x[m] *= f;
  n2 = fmaf(group_sum(squares_of(x), n.group), n.inv_dim, n.eps * f * f);
  return f;
}
// 1 / n, of a scaled head: 0 where n is 0.
__device__ __forceinline__ float inverse_root(float n2) { return n2 == 0.f ? 0.f : 1.f / sqrtf(n2); }

__device__ __forceinline__ float weight_of(const void* w, int64_t i, int f32) {
  return !w ? 1.f : f32 ? ((const float*)w)[i] : Elem<true>::load((const char*)w, i);
}

// The angles of tokens t0 .. t0+nt-1, by all threads.
template <class H>
__device__ __forceinline__ void fill_table(const RotaryArgs& a, const H& head, float2* table, int t0, int nt) {
  for (int j = threadIdx.x; j < nt * a.pairs; j += blockDim.x) {
    const int t = t0 + j / a.pairs, f = j % a.pairs;
    const int p = a.positions ? a.positions[t] : a.live ? a.pos[t & (kMaxSlots - 1)] : a.first + t;
    float c, s;
    turn_of((double)p * a.freq[f], c, s);
    table[head.place_of(j / a.pairs, f)] = float2{c * a.amplitude, s * a.amplitude};
  }
}

// Sums come ahead of the barrier: their branch behind it would hold back the loads out of LDS (38 us for 35 of the case above).
// 7 wavefronts a SIMD: one register more than they leave costs as much.
template <bool BF, bool IL, int UNIT>
__global__ __launch_bounds__(kNormThreads, 7) void norm_rotate_kernel(const NormArgs n) {
  using H = Head<BF, IL, UNIT>;
  const RotaryArgs& a = n.r;
  __shared__ float2 table[H::kTable];
  __shared__ float weights[2][INFS_ROTARY_MAX_DIM];
  __shared__ float exchange[H::kExchange ? kNormThreads * H::kExchangeFloats : 1];
  const int64_t layer = blockIdx.y;
  const int t0 = blockIdx.x * a.tokens_per_wg, nt = min(a.tokens_per_wg, a.tokens - t0);
  const int lane = threadIdx.x & (n.group - 1), first = (int)threadIdx.x >> n.group_log2;
  const int heads = a.q.heads + a.k.heads, total = nt * heads, step = (int)blockDim.x >> n.group_log2;
  const H head(a, lane);
  float* own = exchange + (H::kExchange ? (threadIdx.x - lane) * H::kExchangeFloats : 0);
  const auto place = [&](int i, const char*& in, char*& out, int& t, bool& k) {
    t = divide(i, heads, a.per_head);
    int h = i - t * heads;
    k = h >= a.q.heads;
    const RotaryRows& r = k ? a.k : a.q;
    h -= k ? a.q.heads : 0;
    in = r.in + ((int64_t)(t0 + t) * r.in_row + h * r.in_head + layer * r.in_layer) * H::ES;
    out = r.out + ((int64_t)(t0 + t) * r.out_row + h * r.out_head + layer * r.out_layer) * H::ES;
    return i < total && !(a.live && !((a.live >> ((t0 + t) & 63)) & 1));
  };
  // the first heads are loaded while the angles are computed
  const char* in;
  char* out;
  int t;
  bool k;
  bool there = place(first, in, out, t, k);
  if (!there) t = 0;  // angles of a token that is there
  float x[H::M], y[H::M];
  head.load(in, there, x);
  for (int e = threadIdx.x; e < 2 * INFS_ROTARY_MAX_DIM; e += blockDim.x) {
    const int w = e / INFS_ROTARY_MAX_DIM, i = e % INFS_ROTARY_MAX_DIM;
    if (i < a.head_dim) weights[w][i] = weight_of(n.weight[w], layer * n.weight_layer + i, n.weight_f32);
  }
  fill_table(a, head, table, t0, nt);
  const auto inverse_n = [&] {
    float n2 = fmaf(group_sum(squares_of(x), n.group), n.inv_dim, n.eps);
    if (!__any(out_of_range(n2))) return 1.f / sqrtf(n2);
    scale_heads(x, n2, n);
    return inverse_root(n2);
  };
  float by = inverse_n();
  __syncthreads();
  for (int i = first;;) {
#pragma unroll
    for (int m = 0; m < H::M; ++m) x[m] = x[m] * by * weights[k][head.has(m) ? head.element(m) : 0];
    head.template rotate<false>(table + head.place_of(t, 0), own, x, y);
    head.store(out, there, y);
    i += step;
    if (i - first >= total) break;  // the same for all threads
    there = place(i, in, out, t, k);
    if (!there) t = 0;
    head.load(in, there, x);
    by = inverse_n();
  }
}

// 8192 tokens, 24 heads of 128 in bf16: 37 us for 151 MB (4.1 TB/s), and 4 for d_w's parts in a launch of their own (in
// this one the last work-group would add them behind all others, by a counter that has to be cleared: the workspace is
// the caller's, of any content).
// Work-group (b, y) takes every gridDim.x-th batch of tokens of tensor y of those given, so that a lane's elements
// and their weights stay the same and d_w adds up in registers.
template <bool BF, bool IL, int UNIT>
__global__ __launch_bounds__(kNormThreads) void norm_rotate_grad_kernel(const NormGradArgs n) {
  using H = Head<BF, IL, UNIT>;
  const RotaryArgs& a = n.r;
  __shared__ float2 table[H::kTable];
  __shared__ float shared[kNormThreads * (H::kExchangeFloats > H::M ? H::kExchangeFloats : H::M)];
  const int which = n.first + blockIdx.y;  // 0: q, 1: k
  const RotaryRows& r = which ? a.k : a.q;
  const RotaryRows& up = which ? n.dk : n.dq;
  const int lane = threadIdx.x & (n.group - 1), first = (int)threadIdx.x >> n.group_log2;
  const int heads = r.heads, step = (int)blockDim.x >> n.group_log2, per = n.batch[which];
  const uint32_t per_head = n.per_head[which];
  const H head(a, lane);
  float* own = shared + (threadIdx.x - lane) * H::kExchangeFloats;
  float w[H::M], dw[H::M];
#pragma unroll
  for (int m = 0; m < H::M; ++m) {
    w[m] = head.has(m) ? weight_of(n.weight[which], head.element(m), n.weight_f32) : 0.f;
    dw[m] = 0.f;
  }
  for (int64_t b0 = (int64_t)blockIdx.x * per; b0 < a.tokens; b0 += (int64_t)gridDim.x * per) {
    const int t0 = (int)b0, nt = min(per, a.tokens - t0), total = nt * heads;
    __syncthreads();  // the last batch's angles are no longer read
    fill_table(a, head, table, t0, nt);
    __syncthreads();
    for (int i = first; i - first < total; i += step) {
      const bool there = i < total;
      const int t = there ? divide(i, heads, per_head) : 0, h = there ? i - t * heads : 0;
      float x[H::M], g[H::M], d[H::M];
      const int64_t token = t0 + t;
      head.load(r.in + (token * r.in_row + h * r.in_head) * H::ES, there, x);
      head.load(up.in + (token * up.in_row + h * up.in_head) * H::ES, there, d);
      head.template rotate<true>(table + head.place_of(t, 0), own, d, g);
      const auto along_x = [&] {
        float s = 0.f;
#pragma unroll
        for (int m = 0; m < H::M; ++m)
          if (head.has(m)) s = fmaf(g[m] * w[m], x[m], s);
        return group_sum(s, n.group);
      };
      float n2 = fmaf(group_sum(squares_of(x), n.group), n.inv_dim, n.eps), along = along_x(), f = 1.f;
      float by = 1.f / sqrtf(n2);
      if (__any(out_of_range(n2))) {
        f = scale_heads(x, n2, n);
        by = inverse_root(n2), along = along_x();
      }
      const float back = along * n.inv_dim * by * by;
#pragma unroll
      for (int m = 0; m < H::M; ++m) {
        if (there && head.has(m)) dw[m] = fmaf(g[m], x[m] * by, dw[m]);
        d[m] = by * (g[m] * w[m] - x[m] * back) * f;
      }
      head.store(r.out + (token * r.out_row + h * r.out_head) * H::ES, there, d);
    }
  }
  float* part = n.part + ((int64_t)which * gridDim.x + blockIdx.x) * a.head_dim;
  if (!n.sums[which]) return;
  // over the groups of a wavefront, then over the wavefronts
#pragma unroll
  for (int m = 0; m < H::M; ++m)
    for (int i = n.group; i < 64; i <<= 1) dw[m] += __shfl_xor(dw[m], i);
  __syncthreads();
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) < n.group)
#pragma unroll
    for (int m = 0; m < H::M; ++m) shared[(wave * n.group + lane) * H::M + m] = dw[m];
  __syncthreads();
  if (threadIdx.x < n.group)
#pragma unroll
    for (int m = 0; m < H::M; ++m) {
      float s = dw[m];
      for (int v = 1; v < (int)blockDim.x / 64; ++v) s += shared[(v * n.group + lane) * H::M + m];
      if (head.has(m)) part[head.element(m)] = s;
    }
}

// d_w of tensor y: 32 elements a work-group, parts added by 8 rows of threads and then row by row.
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* part, float* dq, float* dk, int first, int parts,
                                                          int head_dim) {
  __shared__ float rows[8][33];
  const int which = first + blockIdx.y, e = blockIdx.x * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
  float* out = which ? dk : dq;
  if (!out) return;
  const float* p = part + (int64_t)which * parts * head_dim + e;
  float s = 0.f;
  if (e < head_dim)
#pragma unroll 8
    for (int i = row; i < parts; i += 8) s += p[(int64_t)i * head_dim];
  rows[row][threadIdx.x & 31] = s;
  __syncthreads();
  if (row == 0 && e < head_dim) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += rows[i][threadIdx.x];
    out[e] = s;
  }
}

// Whether rows are aligned to 16 bytes (n elements).
bool vector_in(const RotaryRows& r, int n) {
  return r.heads == 0 || ((r.in_row | r.in_head | r.in_layer) % n == 0 && ((uintptr_t)r.in & 15) == 0);
}
bool vector_out(const RotaryRows& r, int n) {
  return r.heads == 0 || ((r.out_row | r.out_head | r.out_layer) % n == 0 && ((uintptr_t)r.out & 15) == 0);
}

// The unit of a call's heads, and the lanes that hold one.
int unit_of(const RotaryArgs& a, bool vector, bool interleaved, int n, int32_t* group, int32_t* group_log2) {
  const int unit = !vector || a.head_dim % n ? kElement : !interleaved && a.pairs % n == 0 ? kPairs : kChunk;
  const int units = unit == kElement ? 64 : unit == kChunk ? a.head_dim / n : (a.head_dim - a.pairs) / n;
  *group_log2 = 0;
  while ((1 << *group_log2) < units) ++*group_log2;
  *group = 1 << *group_log2;
  return unit;
}

uint32_t inverse_of(int n) { return (uint32_t)(((uint64_t(1) << 32) + n - 1) / n); }

#define INFS_NORM(kernel, bf, il) {kernel<bf, il, kElement>, kernel<bf, il, kChunk>, il ? nullptr : kernel<bf, false, kPairs>}
#define INFS_NORMS(kernel) \
  {{INFS_NORM(kernel, false, false), INFS_NORM(kernel, false, true)}, {INFS_NORM(kernel, true, false), INFS_NORM(kernel, true, true)}}

}  // namespace

hipError_t launch_norm_rotate(NormArgs& n, bool bf16, bool interleaved, int layers, hipStream_t stream) {
  RotaryArgs& a = n.r;
  const int heads = a.q.heads + a.k.heads, width = bf16 ? 8 : 4;
  if (a.tokens == 0 || layers == 0 || heads == 0) return hipSuccess;
  const bool vector = vector_in(a.q, width) && vector_out(a.q, width) && vector_in(a.k, width) && vector_out(a.k, width);
  const int unit = unit_of(a, vector, interleaved, width, &n.group, &n.group_log2);
  n.inv_dim = 1.f / a.head_dim;
  a.per_head = inverse_of(heads);
  // tokens of a work-group: one where its heads fill the threads, else as many as do, within the table of angles
  a.tokens_per_wg = (int)std::max<int64_t>(
      1, std::min<int64_t>({kRotaryTable / a.pairs, kRotaryThreads / ((int64_t)heads * n.group), a.tokens}));
  const int threads = (int)std::min<int64_t>(kNormThreads, ((int64_t)heads * a.tokens_per_wg * n.group + 63) / 64 * 64);
  void (*const kernels[2][2][3])(const NormArgs) = INFS_NORMS(norm_rotate_kernel);
  const int64_t per_launch = kMostBlocks / 2 * a.tokens_per_wg;  // tokens of a launch
  for (int64_t left = a.tokens;; left -= per_launch) {
    a.tokens = (int32_t)std::min(per_launch, left);
    const dim3 grid((unsigned)((a.tokens + a.tokens_per_wg - 1) / a.tokens_per_wg), (unsigned)layers);
    hipLaunchKernelGGL(kernels[bf16][interleaved][unit], grid, dim3(threads), 0, stream, n);
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

hipError_t launch_norm_rotate_grad(NormGradArgs& n, bool bf16, bool interleaved, hipStream_t stream) {
  RotaryArgs& a = n.r;
  const int width = bf16 ? 8 : 4;
  const bool vector = vector_in(a.q, width) && vector_out(a.q, width) && vector_in(a.k, width) && vector_out(a.k, width) &&
                      vector_in(n.dq, width) && vector_in(n.dk, width);
  const int unit = unit_of(a, vector, interleaved, width, &n.group, &n.group_log2);
  n.inv_dim = 1.f / a.head_dim;
  n.first = a.q.heads ? 0 : 1;
  const int tensors = (a.q.heads ? 1 : 0) + (a.k.heads ? 1 : 0);
  const int64_t groups = kRotaryThreads >> n.group_log2;
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? a.k.heads : a.q.heads;
    if (!heads) continue;
    n.per_head[i] = inverse_of(heads);
    n.batch[i] = (int)std::max<int64_t>(1, std::min<int64_t>({kRotaryTable / a.pairs, groups / heads, a.tokens}));
  }
  const int parts = norm_grad_parts(a.tokens);
  void (*const kernels[2][2][3])(const NormGradArgs) = INFS_NORMS(norm_rotate_grad_kernel);
  if (parts > 0)
    hipLaunchKernelGGL(kernels[bf16][interleaved][unit], dim3(parts, tensors), dim3(kRotaryThreads), 0, stream, n);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!n.sums[0] && !n.sums[1])) return e;
  hipLaunchKernelGGL(norm_weights_kernel, dim3((a.head_dim + 31) / 32, tensors), dim3(256), 0, stream, n.part, n.sums[0],
                     n.sums[1], n.first, parts, a.head_dim);
  return hipGetLastError();
}

}  // namespace infs
