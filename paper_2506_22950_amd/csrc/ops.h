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

// ---- norms with the rotation ----------------------------------------------------
constexpr int kNormThreads = 512;      // most of a work-group
constexpr int kNormGradParts = 512;    // work-groups a tensor whose sums of d_w are added by a second launch

struct NormWeights {
  const void* weight[2];  // of q and k, or null: ones
  int64_t weight_layer;   // elements
  float eps, inv_dim;     // inv_dim, group: launch_norm_rotate
  int32_t weight_f32, group, group_log2;  // lanes that hold a head
};
struct NormArgs : NormWeights {
  RotaryArgs r;
};
struct NormGradArgs : NormWeights {
  RotaryArgs r;           // in: the rows, out: their gradients
  RotaryRows dq, dk;      // in: gradients of the outputs
  float* sums[2];         // d_w, or null
  float* part;            // [2][parts][head_dim]
  int32_t first, batch[2];  // first tensor; tokens of a batch
  uint32_t per_head[2];
};
static_assert(sizeof(NormGradArgs) <= 4096, "kernel argument block must fit 4 KiB");

inline int norm_grad_parts(int64_t tokens) { return (int)(tokens < kNormGradParts ? tokens : kNormGradParts); }
// Fill in what the structs leave to them.
hipError_t launch_norm_rotate(NormArgs& args, bool bf16, bool interleaved, int layers, hipStream_t stream);
hipError_t launch_norm_rotate_grad(NormGradArgs& args, bool bf16, bool interleaved, hipStream_t stream);
// E_ARG (op_fail), or the weights of every layer.
infs_status pack_norms(const infs_norms* n, NormWeights* out);

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

// ---- the choice of tokens ---------------------------------------------------------
using Sampling = infs_sampling;
constexpr int kChooseMaxRows = 1 << 22;
constexpr int kPieceThreads = 512;
constexpr int kPieceVectors = 8;             // most of a thread, of 16 bytes
constexpr int kChooseSubs = kPieceVectors * kPieceThreads / 64;  // sums of a piece
constexpr int kBins = 1024, kBinsPerOctave = 32;
constexpr int kList = 4096;                  // entries of a row that are ranked
constexpr int kListCount = 1024;             // a top_k whose entries are all listed
constexpr int kChooseRecords = 8192;         // pieces, and ..
constexpr int kChooseRows = 2048;            // .. rows, of a launch
constexpr int kChooseFill = 512;             // pieces that fill the GPU, two a CU
constexpr int kChoosePieces = 2048;          // most of a row

enum RowMode { kDone, kListed, kSums, kLeft };  // what the launch that weighs a row leaves to do
struct RowState {
  float m, lo_bin, hi_bin;  // maximum; bins of the entries to list
  int32_t mode, live;       // RowMode; entries that are not masked
  int32_t pad;
  double whole;             // sum of the weights, in units (by mass)
};
struct PieceState {
  float top;                // NaN: one or +inf in the piece
  int32_t live;             // entries not masked; above the listed bins
  unsigned long long sum;
};

struct ChooseArgs {
  const void* logits;
  int64_t row_stride;  // elements
  const float* uniform;
  const Sampling* each;  // or null: all
  Sampling all;
  int32_t* token;
  float* logprob;  // these two may be null
  int32_t* kept;
  int32_t rows, vocab;
  // launch_choose
  int32_t unit;              // a weight is a number of units of 2^-unit
  int32_t row0;              // of the launch
  int32_t batches, pieces;   // vectors a thread of a piece, pieces of a row
  // The workspace: counters (0 between launches) kCounterStride apart per row, then per row and per piece
  int32_t *arrived, *list_n;
  RowState* state;
  unsigned long long* list;  // [rows][kList]
  PieceState* piece;
  unsigned long long* subs;  // [pieces][kChooseSubs]: sums of a wavefront's 64 vectors
  uint32_t* bins;            // [pieces][kBins]: numbers, or sums of weights
};

// Vectors a thread, pieces of a row, rows of a launch.  Pieces are as small as two a CU allow for all rows together, and
// no larger than the registers hold (top-p of 101 rows of 50257 in fp32: 53 us in 404 pieces, of which some CUs had two
// of the largest, 42 in 505 smaller ones, 60 in 909; 64 rows of 151936 in bf16: 74, 59, 73 in 320, 512, 960).
inline int choose_vectors(int vocab, bool bf16) {  // of a row, at any alignment
  const int n = 16 / (bf16 ? 2 : 4);
  return (vocab + 2 * n - 2) / n;
}
inline int choose_pieces(int vocab, int batches, bool bf16) {
  return (choose_vectors(vocab, bf16) + batches * kPieceThreads - 1) / (batches * kPieceThreads);
}
inline int choose_batches(int rows, int vocab, bool bf16) {
  const int64_t least = choose_pieces(vocab, kPieceVectors, bf16), fill = kChooseFill / (rows < 1 ? 1 : rows);
  const int64_t pieces = fill < least ? least : fill;
  return (int)((choose_vectors(vocab, bf16) + pieces * kPieceThreads - 1) / (pieces * kPieceThreads));
}
inline int choose_rows(int pieces) {
  const int n = kChooseRecords / pieces;
  return n < 1 ? 1 : n < kChooseRows ? n : kChooseRows;
}


hipError_t launch_choose(ChooseArgs& args, bool bf16, hipStream_t stream);

// ---- attention of packed sequences ------------------------------------------------
// Work-groups of a launch: of at most 512 threads, so half as many as of 256.
constexpr int64_t kAttendMostBlocks = kMostBlocks / 2;

struct AttendShape {
  const int32_t *q_offsets, *k_offsets;  // [sequences + 1]
  int32_t sequences, q_tokens, k_tokens, q_heads, kv_heads, hpk;
  uint32_t hpk_inv;                      // 2^32 / hpk, rounded up
  float scale;
  // Walks that several work-groups share: their parts' results, and how many have come (zero between launches).
  float* part;
  int32_t* arrived;
  int32_t parts, slots;  // launch_attend, launch_attend_grad
};
constexpr int kAttendParts = 512;                  // work-groups of a launch with shared walks
constexpr int kAttendPartFloats = 2 * 32;  // of an element of the head: two results (or one with a maximum and a sum)
                                           // of 32 rows

struct AttendArgs : AttendShape {
  const char *q, *k, *v;
  char* o;
  float* lse;  // [q_tokens, q_heads], or null
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;  // bytes
};

struct AttendGradArgs : AttendShape {
  const char *q, *k, *v, *o, *d_o;
  char *dq, *dk, *dv;
  const float* lse;
  float* delta;  // [q_tokens, q_heads]: d_o.o of every row
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, do_row, do_head, dq_row, dq_head, dk_row, dk_head,
      dv_row, dv_head;           // bytes
};

hipError_t launch_attend(AttendArgs& args, bool bf16, int head_dim, hipStream_t stream);
hipError_t launch_attend_grad(AttendGradArgs& args, bool bf16, int head_dim, hipStream_t stream);

}  // namespace infs
