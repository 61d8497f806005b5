// Responses' pages: forks, and dense rows to and from pages.
//
// A page holds kPageTokens tokens of every KV head: [head][K | V][page of a head].
// fp32 pages are token rows.  bf16 and E4M3 pages are in MFMA operand order (see
// RespMfma): K unit (kb, lane) = 8 dims 32kb + 8(lane/16) + e of token lane % 16; V
// unit (db, lane) = dim 16db + lane % 16 of the 4 tokens 4(lane/16) + e.  So a K
// unit is 16 bytes of a dense bf16 row, while 8 V units of neighbouring dims are an
// 8 x 4 block of elements to transpose, which a lane does in its registers.
//
// Bound by memory: every element is read and written once.  A wavefront (head size
// 128) or half of one (64) takes a page of one KV head: 4 KiB of K and V each in
// bf16, eight loads of 16 bytes a lane in flight.  5804 tokens of eight responses, 28
// layers, 8 heads of 128 in and out again move 2.0 GB (E4M3) in 367 us and 2.66 GB
// (bf16) in 491 us: 5.4 TB/s, the rate of a large copy.  Loads or stores past the
// caches make one direction faster and the next as much slower; in fp32 both
// together gain from storing past them (481 against 514 us for 2.66 GB).
#include "decode.h"
#include "ops.h"

namespace infs {
namespace {

constexpr int kMoveThreads = 256;

template <int BF, int K8, int D>
struct Page {
  static constexpr int KES = K8 ? 1 : BF ? 2 : 4;            // stored element
  static constexpr int ES = BF ? 2 : 4;                      // element of a dense row
  static constexpr int N = 16 / ES;                          // elements of 16 bytes of a dense row
  static constexpr int HALF = kPageTokens * D * KES;         // K (or V) of one head
  static constexpr int LANES = D / 2;                        // lanes that move a page of one head
  static constexpr int CHUNKS = D / N;                       // 16-byte chunks of a row
  static constexpr int ROUNDS = kPageTokens * CHUNKS / LANES;
  static constexpr int GROUPS = kMoveThreads / LANES;
};

// Elements of token pairs of dims (2k, 2k + 1): the low or the high halves of two words.
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

__device__ __forceinline__ u32x2 widen4(uint32_t w) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true))};
}

// One page of one head, tokens below n (of 16) to dense rows: row 0 of K and V, rows `pitch` bytes apart.
template <int BF, int K8, int D>
__device__ __forceinline__ void page_to_rows(const char* page, char* k, char* v, int64_t pitch, int n, int lane) {
  using P = Page<BF, K8, D>;
  if constexpr (!BF) {
    u32x4 x[2][P::ROUNDS];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
      for (int i = 0; i < P::ROUNDS; ++i)
        x[kind][i] = __builtin_nontemporal_load((const u32x4*)(page + kind * P::HALF) + i * P::LANES + lane);
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
      for (int i = 0; i < P::ROUNDS; ++i) {
        const int at = i * P::LANES + lane, t = at / P::CHUNKS, c = at % P::CHUNKS;
        if (t < n) __builtin_nontemporal_store(x[kind][i], (u32x4*)((kind ? v : k) + t * pitch + c * 16));
      }
  } else {
    u32x4 kx[P::ROUNDS], rows[4];
#pragma unroll
    for (int i = 0; i < P::ROUNDS; ++i) {
      const int at = i * P::LANES + lane, t = at / P::CHUNKS, c = at % P::CHUNKS;
      const char* unit = page + ((c >> 2) * 64 + (c & 3) * 16 + t) * 8 * P::KES;
      if constexpr (K8)
        kx[i] = widen_e4m3(*(const uint2*)unit);
      else
        kx[i] = *(const u32x4*)unit;
    }
    const int q = lane / P::CHUNKS, o = lane % P::CHUNKS;  // tokens 4q .. 4q+3, dims 8o .. 8o+7
    u32x2 u[8];
    {
      const u32x4* unit = (const u32x4*)(page + P::HALF + ((o >> 1) * 64 + q * 16 + (o & 1) * 8) * 4 * P::KES);
      if constexpr (K8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x4 w = unit[i];
#pragma unroll
          for (int j = 0; j < 4; ++j) u[4 * i + j] = widen4(w[j]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 w = unit[i];
          u[2 * i] = u32x2{w[0], w[1]};
          u[2 * i + 1] = u32x2{w[2], w[3]};
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        rows[e][j] = (e & 1) ? high_halves(u[2 * j][e >> 1], u[2 * j + 1][e >> 1])
                             : low_halves(u[2 * j][e >> 1], u[2 * j + 1][e >> 1]);
#pragma unroll
    for (int i = 0; i < P::ROUNDS; ++i) {
      const int at = i * P::LANES + lane, t = at / P::CHUNKS, c = at % P::CHUNKS;
      if (t < n) *(u32x4*)(k + t * pitch + c * 16) = kx[i];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * q + e < n) *(u32x4*)(v + (4 * q + e) * pitch + o * 16) = rows[e];
  }
}

// The other way; the page's tokens from n on become zero.
template <int BF, int K8, int D>
__device__ __forceinline__ void rows_to_page(char* page, const char* k, const char* v, int64_t pitch, int n, int lane) {
  using P = Page<BF, K8, D>;
  const u32x4 zero = {0, 0, 0, 0};
  if constexpr (!BF) {
    u32x4 x[2][P::ROUNDS];
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
      for (int i = 0; i < P::ROUNDS; ++i) {
        const int at = i * P::LANES + lane, t = at / P::CHUNKS, c = at % P::CHUNKS;
        x[kind][i] = t < n ? *(const u32x4*)((kind ? v : k) + t * pitch + c * 16) : zero;
      }
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
      for (int i = 0; i < P::ROUNDS; ++i) *((u32x4*)(page + kind * P::HALF) + i * P::LANES + lane) = x[kind][i];
  } else {
    u32x4 kx[P::ROUNDS], rows[4];
    const int q = lane / P::CHUNKS, o = lane % P::CHUNKS;
#pragma unroll
    for (int i = 0; i < P::ROUNDS; ++i) {
      const int at = i * P::LANES + lane, t = at / P::CHUNKS, c = at % P::CHUNKS;
      kx[i] = t < n ? *(const u32x4*)(k + t * pitch + c * 16) : zero;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) rows[e] = 4 * q + e < n ? *(const u32x4*)(v + (4 * q + e) * pitch + o * 16) : zero;
#pragma unroll
    for (int i = 0; i < P::ROUNDS; ++i) {
      const int at = i * P::LANES + lane, t = at / P::CHUNKS, c = at % P::CHUNKS;
      char* unit = page + ((c >> 2) * 64 + (c & 3) * 16 + t) * 8 * P::KES;
      if constexpr (K8)
        *(uint2*)unit = narrow_e4m3(kx[i]);
      else
        *(u32x4*)unit = kx[i];
    }
    u32x2 u[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[2 * j] = u32x2{low_halves(rows[0][j], rows[1][j]), low_halves(rows[2][j], rows[3][j])};
      u[2 * j + 1] = u32x2{high_halves(rows[0][j], rows[1][j]), high_halves(rows[2][j], rows[3][j])};
    }
    u32x4* unit = (u32x4*)(page + P::HALF + ((o >> 1) * 64 + q * 16 + (o & 1) * 8) * 4 * P::KES);
    if constexpr (K8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = narrow4_e4m3(u[4 * i + j].x, u[4 * i + j].y);
        unit[i] = w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) unit[i] = u32x4{u[2 * i].x, u[2 * i].y, u[2 * i + 1].x, u[2 * i + 1].y};
    }
  }
}

template <int BF, int K8, int D, bool OUT>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(const MoveArgs a) {
  using P = Page<BF, K8, D>;
  int i = 0;
  while (i + 1 < a.n && (int)blockIdx.x >= a.r[i + 1].first_block) ++i;
  const MoveArgs::Response& r = a.r[i];
  const int group = ((int)blockIdx.x - r.first_block) * P::GROUPS + (int)threadIdx.x / P::LANES;
  const int page = group / a.hkv, head = group - page * a.hkv;
  if (page * kPageTokens >= r.len) return;
  const int64_t layer = blockIdx.y, pitch = (int64_t)a.hkv * D * P::ES;
  const int64_t stride = a.layer_stride ? a.layer_stride : r.len * pitch;
  const int64_t row = layer * stride + (int64_t)page * kPageTokens * pitch + head * (D * P::ES);
  int32_t* entry = a.page_table + (int64_t)r.seq * a.pages_per_slot + page;
  int64_t pg = 0;
  if (r.runs > 0) {
    for (int j = r.first_run; j < r.first_run + r.runs; ++j) {
      const int d = page - a.run[j].at;
      if (d >= 0 && d < a.run[j].count) pg = a.run[j].page + d;
    }
    if (layer == 0 && head == 0 && threadIdx.x % P::LANES == 0) *entry = (int32_t)pg;
  } else {
    pg = *entry;
  }
  char* at = a.pool + layer * a.layer_bytes + (pg * a.hkv + head) * (2 * P::HALF);
  const int n = min(kPageTokens, r.len - page * kPageTokens), lane = (int)threadIdx.x % P::LANES;
  if constexpr (OUT)
    page_to_rows<BF, K8, D>(at, r.k + row, r.v + row, pitch, n, lane);
  else
    rows_to_page<BF, K8, D>(at, r.k + row, r.v + row, pitch, n, lane);
}

// A part of a page is copied whole: the source's tokens behind the part come along,
// and every kernel that reads the page clears what lies behind its response's end.
constexpr int kForkThreads = 256;
constexpr int kForkUnits = 4;  // 16-byte units of a thread

__global__ __launch_bounds__(kForkThreads) void fork_kernel(const ForkArgs a) {
  const ForkArgs::Fork& f = a.fork[blockIdx.y];
  const int64_t layer = blockIdx.z;
  if (layer == 0 && blockIdx.x == 0) {
    const int32_t* src = a.page_table + (int64_t)f.src_seq * a.pages_per_slot;
    int32_t* dst = a.page_table + (int64_t)f.dst_seq * a.pages_per_slot;
    for (int i = threadIdx.x; i < f.full; i += kForkThreads) dst[i] = src[i];
    if (threadIdx.x == 0 && f.dst_page >= 0) dst[f.full] = f.dst_page;
  }
  if (f.dst_page < 0) return;
  const u32x4* from = (const u32x4*)(a.pool + layer * a.layer_bytes + f.src_page * a.page_bytes);
  u32x4* to = (u32x4*)(a.pool + layer * a.layer_bytes + f.dst_page * a.page_bytes);
  const int units = (int)(a.page_bytes / 16), u0 = (int)blockIdx.x * (kForkThreads * kForkUnits) + (int)threadIdx.x;
  u32x4 x[kForkUnits];
#pragma unroll
  for (int i = 0; i < kForkUnits; ++i)
    if (u0 + i * kForkThreads < units) x[i] = from[u0 + i * kForkThreads];
#pragma unroll
  for (int i = 0; i < kForkUnits; ++i)
    if (u0 + i * kForkThreads < units) to[u0 + i * kForkThreads] = x[i];
}

__global__ __launch_bounds__(64) void page_runs_kernel(const PageRuns a) {
  const PageRun& r = a.run[blockIdx.x];
  for (int i = threadIdx.x; i < r.count; i += 64) a.page_table[r.at + i] = r.page + i;
}

template <int BF, int K8, int D, bool OUT>
hipError_t launch_move(MoveArgs& a, int layers, hipStream_t stream) {
  using P = Page<BF, K8, D>;
  int blocks = 0;
  for (int i = 0; i < a.n; ++i) {
    a.r[i].first_block = blocks;
    blocks += ((a.r[i].len + kPageTokens - 1) / kPageTokens * a.hkv + P::GROUPS - 1) / P::GROUPS;
  }
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL((move_kernel<BF, K8, D, OUT>), dim3(blocks, layers), dim3(kMoveThreads), 0, stream, a);
  return hipGetLastError();
}

template <bool OUT>
hipError_t launch_move(const PageFormat& f, MoveArgs& a, int layers, hipStream_t stream) {
  if (f.kv8) return f.head_dim == 128 ? launch_move<1, 1, 128, OUT>(a, layers, stream) : hipErrorInvalidValue;
  if (f.bf16)
    return f.head_dim == 128 ? launch_move<1, 0, 128, OUT>(a, layers, stream) : launch_move<1, 0, 64, OUT>(a, layers, stream);
  return f.head_dim == 128 ? launch_move<0, 0, 128, OUT>(a, layers, stream) : launch_move<0, 0, 64, OUT>(a, layers, stream);
}

}  // namespace

hipError_t launch_fork(const ForkArgs& a, int layers, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  const int units = (int)(a.page_bytes / 16), per = kForkThreads * kForkUnits;
  hipLaunchKernelGGL(fork_kernel, dim3((units + per - 1) / per, a.n, layers), dim3(kForkThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_page_runs(const PageRuns& a, hipStream_t stream) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(page_runs_kernel, dim3(a.n), dim3(64), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_export(const PageFormat& f, MoveArgs& a, int layers, hipStream_t stream) {
  return launch_move<true>(f, a, layers, stream);
}
hipError_t launch_import(const PageFormat& f, MoveArgs& a, int layers, hipStream_t stream) {
  return launch_move<false>(f, a, layers, stream);
}

}  // namespace infs
