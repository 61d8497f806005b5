// Launch entry points of the row and page operators (rotary.hip, score.hip,
// pages.hip), and the error and device helpers their host code shares.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "infs.h"
#include "plan.h"

// Host only: the frequencies a rotary configuration gives.
struct infs_rotary {
  infs_rotary_config cfg{};
  int pairs = 0;
  double freq[INFS_ROTARY_MAX_DIM / 2] = {};  // angle per position of pair j
  double amplitude = 1.0;
};

namespace infs {

// Records the message infs_last_error(NULL) gives on this thread; returns st.
infs_status op_fail(infs_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// Makes the device of `stream` current for its lifetime (the null stream: device `fallback`, or
// the current one where that is -1).
class StreamDevice {
 public:
  explicit StreamDevice(hipStream_t stream, int fallback = -1) {
    int dev = fallback;
    if (!stream && dev < 0) return;
    status_ = hipGetDevice(&before_);
    if (status_ == hipSuccess && stream) status_ = hipStreamGetDevice(stream, &dev);
    if (status_ == hipSuccess && dev != before_) {
      status_ = hipSetDevice(dev);
      changed_ = status_ == hipSuccess;
    }
  }
  ~StreamDevice() {
    if (changed_) (void)hipSetDevice(before_);
  }
  StreamDevice(const StreamDevice&) = delete;
  StreamDevice& operator=(const StreamDevice&) = delete;
  hipError_t status() const { return status_; }

 private:
  int before_ = 0;
  bool changed_ = false;
  hipError_t status_ = hipSuccess;
};

// Work-groups of 256 threads of one launch: a grid's threads along an axis are counted in 32 bits.
constexpr int64_t kMostBlocks = int64_t(1) << 23;

// ---- rotary positions --------------------------------------------------------
constexpr int kRotaryThreads = 256;    // most of a work-group (see launch_rotate)
constexpr int kRotaryFewBlocks = 256;
constexpr int kRotaryTable = 256;  // angles of a work-group
static_assert(INFS_ROTARY_MAX_DIM / 2 <= kRotaryTable, "a token's pairs fit the table");

struct RotaryRows {
  const char* in;
  char* out;
  int64_t in_row, in_head, in_layer, out_row, out_head, out_layer;  // elements
  int32_t heads;                                                    // 0: no such rows
};

struct RotaryArgs {
  double freq[INFS_ROTARY_MAX_DIM / 2];
  RotaryRows q, k;
  const int32_t* positions;  // or null: pos[] of the slots (live != 0), else first + token
  uint64_t live;             // slots: bit t set where token t is rotated (0: every token)
  int32_t tokens, first, head_dim, pairs;
  int32_t tokens_per_wg;     // tokens_per_wg * pairs <= kRotaryTable
  uint32_t per_unit, per_head;  // 2^32 over the units of a head and over the heads, rounded up
  float amplitude, sign;     // of cos and sin; sign of the angle
  int32_t pos[kMaxSlots];
};
static_assert(sizeof(RotaryArgs) <= 4096, "kernel argument block must fit 4 KiB");

// Rotate `layers` layers of rows; fills in tokens_per_wg, per_unit and per_head.
hipError_t launch_rotate(RotaryArgs& args, bool bf16, bool interleaved, int layers, hipStream_t stream);

// Checks and packs one side's rows (op_fail on E_ARG).  es: element bytes.
infs_status pack_rotary_rows(const infs_rows* r, const char* what, int head_dim, int64_t tokens, int layers, size_t es,
                             RotaryRows* out);
// The configuration's part of the launch arguments.
void set_rotary(const infs_rotary& r, bool inverse, RotaryArgs* a);

// ---- scores of tokens -----------------------------------------------------------
constexpr int kScoreMaxRows = 1 << 23;
static_assert(kScoreMaxRows <= kMostBlocks, "a work-group a row");
constexpr int kScoreMaxPieces = 32;      // pieces of a row
constexpr int kScorePieceKeys = 64;      // candidates that a piece hands over
constexpr int kScorePartStride = 32;     // floats: no two work-groups write one 128-byte line
constexpr int kScoreWaveRows = 2048;     // rows from which ..
constexpr int kScoreWaveVectors = 1024;  // .. rows of so many 16-byte vectors go a wavefront each

struct ScoreArgs {
  const void* logits;
  int64_t row_stride;  // elements
  const int32_t* tokens;
  float* logprob;      // [rows]; these five may be null
  float* entropy;      // [rows]
  int32_t* top_id;     // [rows, top_k]
  float* top_logprob;  // [rows, top_k]
  float* stats;        // [rows, 2]
  int32_t rows, vocab, top_k;
  float inv_t;         // 1 / temperature
  int32_t wave_rows;        // 1: a wavefront a row (plan_score); else
  int32_t pieces, batches;  // pieces of a row, batches of a piece
  int32_t resident;         // work-groups that fit the GPU at once (score_resident), the same whatever outputs are
                            // asked for: rows are cut, and sums rounded, alike
  // Where rows are cut (pieces > 1), per record row * pieces + piece: the part of a piece (3 floats,
  // kScorePartStride apart) and its candidates [kScorePieceKeys]; and, kCounterStride apart, the pieces
  // of a row that have arrived (0 between launches).
  float* part;
  unsigned long long* keys;
  int32_t* arrived;
};
// Rows are cut only where that leaves at most this many records.
constexpr int kScoreMaxRecords = 2048;

struct ScoreGradArgs {
  const void* logits;
  void* grad;
  int64_t row_stride, grad_row_stride;
  const int32_t* tokens;     // null where d_logprob is
  const float* stats;
  const float* entropy;      // null where d_entropy is
  const float* d_logprob;
  const float* d_entropy;
  int32_t rows, vocab;
  float inv_t;
  int32_t batches;           // of a row (launch_score_grad)
};

// Work-groups of the forward kernel that the current device keeps resident at once.
hipError_t score_resident(bool bf16, bool top, int* resident);

// Fills in wave_rows, pieces and batches.
hipError_t launch_score(ScoreArgs& args, bool bf16, hipStream_t stream);
// The workspace of a scorer: arrived, part, then (top) keys.
constexpr size_t kScoreArrivedBytes = sizeof(int32_t) * kCounterStride * kScoreMaxRecords;
constexpr size_t kScorePartBytes = sizeof(float) * kScorePartStride * kScoreMaxRecords;
constexpr size_t kScoreKeyBytes = sizeof(unsigned long long) * kScorePieceKeys * kScoreMaxRecords;
hipError_t launch_score_grad(ScoreGradArgs& args, bool bf16, hipStream_t stream);

// ---- responses' pages -----------------------------------------------------------
struct ForkArgs {
  char* pool;
  int64_t layer_bytes, page_bytes;  // of the pool's layers, of a page (all KV heads, K and V)
  int32_t* page_table;
  int32_t pages_per_slot, n;
  struct Fork {
    int32_t src_seq, dst_seq;  // page-table rows
    int32_t full;              // pages shared
    int32_t src_page, dst_page;  // a part of a page is copied (dst_page >= 0)
  } fork[kMaxSlots];
};
static_assert(sizeof(ForkArgs) <= 4096, "kernel argument block must fit 4 KiB");

// Pages that follow each other: entries at .. at+count-1 of a list are page, page+1, ...
struct PageRun {
  int32_t at, page, count;
};

// Runs to write into the page table (at: its entries).
constexpr int kRunsPerLaunch = 300;
struct PageRuns {
  int32_t* page_table;
  int32_t n;
  PageRun run[kRunsPerLaunch];
};
static_assert(sizeof(PageRuns) <= 4096, "kernel argument block must fit 4 KiB");

// Dense rows <-> pages of several responses.
constexpr int kRunsInline = 96;
struct MoveArgs {
  char* pool;
  int64_t layer_bytes, layer_stride;  // layer_stride 0: a response's own rows
  int32_t* page_table;
  int32_t pages_per_slot, hkv, n;
  struct Response {
    char *k, *v;
    int32_t seq, len;
    int32_t first_block;       // first work-group of the response in a layer
    int16_t first_run, runs;   // its runs (at: its pages); 0 runs: its pages are in the page table
  } r[kMaxSlots];
  PageRun run[kRunsInline];    // import: pages taken in this call, which it writes into the page table
};
static_assert(sizeof(MoveArgs) <= 4096, "kernel argument block must fit 4 KiB");

// How responses lie in pages (KernelKey's bf16 and kv8, head_dim).
struct PageFormat {
  int bf16, kv8, head_dim;
};

hipError_t launch_fork(const ForkArgs& args, int layers, hipStream_t stream);
hipError_t launch_page_runs(const PageRuns& args, hipStream_t stream);
// Fills in first_block.
hipError_t launch_export(const PageFormat& f, MoveArgs& args, int layers, hipStream_t stream);
hipError_t launch_import(const PageFormat& f, MoveArgs& args, int layers, hipStream_t stream);

}  // namespace infs
