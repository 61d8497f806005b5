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

namespace infs {
namespace {

constexpr int kThreads = 256;
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
__device__ __forceinline__ Part join(const Part& a, const Part& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float da = fmaxf((a.m - m) * c, kFar), db = fmaxf((b.m - m) * c, kFar);
  const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
  return Part{m, a.s * ea + b.s * eb, (a.w + a.s * da) * ea + (b.w + b.s * db) * eb};
}

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

// One work-group a row; every alternative is a pass of its own over the row.
template <bool BF>
__global__ __launch_bounds__(kThreads) void score_kernel(const ScoreArgs a) {
  const int64_t row = blockIdx.x;
  const char* z = (const char*)a.logits + row * a.row_stride * (BF ? 2 : 4);
  const float c = a.inv_t * kLog2E;
  Part p = empty_part();
  for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
    const float x = load1<BF>(z, i), m = fmaxf(p.m, x);
    const float y = (x - m) * c, d = fmaxf((p.m - m) * c, kFar), e = __builtin_amdgcn_exp2f(y), f = __builtin_amdgcn_exp2f(d);
    p.w = (p.w + p.s * d) * f + e * fmaxf(y, kFar);
    p.s = p.s * f + e;
    p.m = m;
  }
  __shared__ Part parts[kThreads];
  __shared__ unsigned long long best[kThreads];
  parts[threadIdx.x] = p;
  __syncthreads();
  for (int n = kThreads / 2; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) parts[threadIdx.x] = join(parts[threadIdx.x], parts[threadIdx.x + n], c);
    __syncthreads();
  }
  p = parts[0];
  const bool none = p.s == 0.f;  // every entry masked
  const float log2_s = log2f(p.s), ln_s = none ? -__builtin_huge_valf() : log2_s * kLn2;
  if (threadIdx.x == 0) {
    if (a.logprob) {
      const int t = a.tokens[row];
      float lp = __builtin_nanf("");
      if (t == -1)
        lp = 0.f;
      else if (t >= 0 && t < a.vocab)
        lp = none ? -__builtin_huge_valf() : (load1<BF>(z, t) - p.m) * a.inv_t - ln_s;
      a.logprob[row] = lp;
    }
    if (a.entropy) a.entropy[row] = none ? 0.f : kLn2 * (log2_s - p.w / p.s);
    if (a.stats) {
      a.stats[2 * row] = none ? -__builtin_huge_valf() : p.m;
      a.stats[2 * row + 1] = ln_s;
    }
  }
  if (!a.top_id) return;
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.top_k; ++k) {
    unsigned long long b = 0;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
      const unsigned long long key = key_of(load1<BF>(z, i), i);
      if (key < last && key > b) b = key;
    }
    __syncthreads();
    best[threadIdx.x] = b;
    __syncthreads();
    for (int n = kThreads / 2; n > 0; n >>= 1) {
      if ((int)threadIdx.x < n && best[threadIdx.x + n] > best[threadIdx.x]) best[threadIdx.x] = best[threadIdx.x + n];
      __syncthreads();
    }
    last = best[0];
    if (threadIdx.x == 0) {
      const bool bad = !(p.s == p.s);
      a.top_id[row * a.top_k + k] = last == 0 || bad ? -1 : key_id(last);
      a.top_logprob[row * a.top_k + k] =
          bad ? __builtin_nanf("") : last == 0 ? -__builtin_huge_valf() : (key_value(last) - p.m) * a.inv_t - ln_s;
    }
  }
}

// grad_j = p_j (A + B log p_j) + [j = token] C with A = -(g_lp + g_h H) / T, B = -g_h / T,
// C = g_lp / T.  Rows from rows on are no work: a work-group strides over them.
template <bool BF>
__global__ __launch_bounds__(kThreads) void score_grad_kernel(const ScoreGradArgs a) {
  const float c = a.inv_t * kLog2E;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const char* z = (const char*)a.logits + row * a.row_stride * (BF ? 2 : 4);
    char* g = (char*)a.grad + row * a.grad_row_stride * (BF ? 2 : 4);
    const float m = a.stats[2 * row], ls2 = a.stats[2 * row + 1] * kLog2E;
    const int t = a.d_logprob ? a.tokens[row] : -1;
    float g_lp = a.d_logprob && t != -1 ? a.d_logprob[row] : 0.f;
    if (t < -1 || t >= a.vocab) g_lp = __builtin_nanf("");
    const float g_h = a.d_entropy ? a.d_entropy[row] : 0.f, h = a.d_entropy ? a.entropy[row] : 0.f;
    const float ca = -(g_lp + g_h * h) * a.inv_t, cb = -g_h * a.inv_t * kLn2, cc = g_lp * a.inv_t;
    const bool none = m == -__builtin_huge_valf();
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.vocab; i += gridDim.x * kThreads) {
      const float y = (load1<BF>(z, i) - m) * c - ls2, p = __builtin_amdgcn_exp2f(y);
      float r = p * (ca + cb * fmaxf(y, kFar));
      if (i == t) r += cc;
      store1<BF>(g, i, none ? 0.f : r);
    }
  }
}

}  // namespace

hipError_t launch_score(const ScoreArgs& a, bool bf16, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(bf16 ? score_kernel<true> : score_kernel<false>, dim3(a.rows), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_score_grad(const ScoreGradArgs& a, bool bf16, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  const unsigned x = (unsigned)((a.vocab + kThreads - 1) / kThreads), y = (unsigned)(a.rows < 32768 ? a.rows : 32768);
  hipLaunchKernelGGL(bf16 ? score_grad_kernel<true> : score_grad_kernel<false>, dim3(x < 64 ? x : 64, y), dim3(kThreads), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace infs
