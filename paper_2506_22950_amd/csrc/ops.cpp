// Host side of the operators that need no context: rotary configurations and
// rows, and scores of tokens.  Arguments are checked before anything is
// enqueued; messages go to infs_last_error(NULL) of the calling thread.
#include "ops.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <new>

namespace infs {

infs_status pack_rotary_rows(const infs_rows* r, const char* what, int head_dim, int64_t tokens, int layers, size_t es,
                             RotaryRows* out) {
  *out = RotaryRows{};
  if (r->heads < 1 || r->heads > 4096) return op_fail(INFS_E_ARG, "%s: heads must be in [1, 4096]", what);
  const int64_t s[6] = {r->in_row, r->in_head, r->in_layer, r->out_row, r->out_head, r->out_layer};
  for (int64_t x : s)
    if (x < 0 || x > (int64_t(1) << 40)) return op_fail(INFS_E_ARG, "%s: strides must be in [0, 2^40] elements", what);
  const int64_t head = head_dim, row = head * r->heads, layer = row * tokens;
  out->in_head = r->in_head ? r->in_head : head;
  out->in_row = r->in_row ? r->in_row : row;
  out->in_layer = r->in_layer ? r->in_layer : layer;
  out->out_head = r->out_head ? r->out_head : head;
  out->out_row = r->out_row ? r->out_row : row;
  out->out_layer = r->out_layer ? r->out_layer : layer;
  // strides of axes longer than one: heads may not overlap
  if ((r->heads > 1 && (out->in_head < head || out->out_head < head)) ||
      (tokens > 1 && (out->in_row < head || out->out_row < head)) ||
      (layers > 1 && (out->in_layer < head || out->out_layer < head)))
    return op_fail(INFS_E_ARG, "%s: strides below one head's %d elements", what, head_dim);
  if (((uintptr_t)r->in | (uintptr_t)r->out) % es) return op_fail(INFS_E_ARG, "%s: rows must be aligned to an element", what);
  if (r->in == r->out && ((r->heads > 1 && out->in_head != out->out_head) || (tokens > 1 && out->in_row != out->out_row) ||
                          (layers > 1 && out->in_layer != out->out_layer)))
    return op_fail(INFS_E_ARG, "%s: rows rotated in place need equal strides", what);
  out->in = (const char*)r->in;
  out->out = (char*)r->out;
  out->heads = r->heads;
  return INFS_OK;
}

void set_rotary(const infs_rotary& r, bool inverse, RotaryArgs* a) {
  std::copy(r.freq, r.freq + r.pairs, a->freq);
  a->head_dim = r.cfg.head_dim;
  a->pairs = r.pairs;
  a->amplitude = (float)r.amplitude;
  a->sign = inverse ? -1.f : 1.f;
}

}  // namespace infs

using infs::op_fail;

struct infs_scorer {
  infs_scorer_config cfg{};
  bool dry = false, bf16 = false;
  size_t es = 0;
  float inv_t = 1.f;
  hipStream_t stream = nullptr;
  int device = 0;
  int resident = 0;  // work-groups on the GPU at once, of the kernel that gives all outputs of the scorer
  // Arrivals, parts and candidates of the pieces of rows (see ScoreArgs), zero before the first launch.
  char* workspace = nullptr;
};

namespace {

infs_status check_rows(const infs_scorer* s, int32_t rows, const void* logits, int64_t* stride, const char* what) {
  if (rows < 0 || rows > s->cfg.max_rows) return op_fail(INFS_E_ARG, "rows must be in [0, %d]", s->cfg.max_rows);
  if (*stride == 0) *stride = s->cfg.vocab;
  if (*stride < s->cfg.vocab || *stride > (int64_t(1) << 40))
    return op_fail(INFS_E_ARG, "%s: row stride must be 0 or in [vocab, 2^40]", what);
  if (rows > 0 && !s->dry && !logits) return op_fail(INFS_E_ARG, "%s: null buffer", what);
  if ((uintptr_t)logits % s->es) return op_fail(INFS_E_ARG, "%s must be aligned to an element", what);
  return INFS_OK;
}

size_t workspace_bytes(const infs_scorer& s) {
  return infs::kScoreArrivedBytes + infs::kScorePartBytes + (s.cfg.top_k > 0 ? infs::kScoreKeyBytes : 0);
}

bool misaligned(std::initializer_list<const void*> ptrs, size_t n) {
  for (const void* p : ptrs)
    if ((uintptr_t)p % n) return true;
  return false;
}

}  // namespace

extern "C" {

infs_status infs_rotary_create(const infs_rotary_config* cfg, infs_rotary** out) {
  if (!out) return op_fail(INFS_E_ARG, "out is null");
  *out = nullptr;
  if (!cfg) return op_fail(INFS_E_ARG, "cfg is null");
  const infs_rotary_config& k = *cfg;
  if (k.head_dim < 2 || k.head_dim > INFS_ROTARY_MAX_DIM)
    return op_fail(INFS_E_ARG, "head_dim must be in [2, %d]", INFS_ROTARY_MAX_DIM);
  if (k.rotary_dim < 2 || k.rotary_dim > k.head_dim || k.rotary_dim % 2)
    return op_fail(INFS_E_ARG, "rotary_dim must be even and in [2, head_dim]");
  if (k.layout != INFS_ROTARY_HALF && k.layout != INFS_ROTARY_INTERLEAVED)
    return op_fail(INFS_E_ARG, "layout must be INFS_ROTARY_HALF or INFS_ROTARY_INTERLEAVED");
  if (k.scaling < INFS_ROTARY_NONE || k.scaling > INFS_ROTARY_BANDS) return op_fail(INFS_E_ARG, "unknown scaling");
  if (!(k.base > 1.0) || !std::isfinite(k.base)) return op_fail(INFS_E_ARG, "base must be finite and above 1");
  const bool scaled = k.scaling != INFS_ROTARY_NONE, ramped = k.scaling == INFS_ROTARY_YARN || k.scaling == INFS_ROTARY_BANDS;
  if (scaled && (!(k.factor >= 1.0) || !std::isfinite(k.factor)))
    return op_fail(INFS_E_ARG, "factor must be finite and at least 1");
  if (k.scaling == INFS_ROTARY_NTK && k.rotary_dim < 4)
    return op_fail(INFS_E_ARG, "INFS_ROTARY_NTK needs a rotary_dim of at least 4");
  if (ramped && k.trained_len < 1) return op_fail(INFS_E_ARG, "trained_len must be at least 1");
  if (ramped && (!(k.low > 0.0) || !(k.high > k.low) || !std::isfinite(k.high)))
    return op_fail(INFS_E_ARG, "low and high must be finite with 0 < low < high");
  if (!(k.amplitude >= 0.0) || !std::isfinite(k.amplitude))
    return op_fail(INFS_E_ARG, "amplitude must be finite and >= 0");
  infs_rotary* r = new (std::nothrow) infs_rotary;
  if (!r) return op_fail(INFS_E_NOMEM, "host allocation failed");
  r->cfg = k;
  r->pairs = k.rotary_dim / 2;
  const double rd = k.rotary_dim, s = scaled ? k.factor : 1.0, two_pi = 6.283185307179586476925;
  const double base = k.scaling == INFS_ROTARY_NTK ? k.base * std::pow(s, rd / (rd - 2.0)) : k.base;
  // YARN: the pair index whose frequency makes `turns` turns over the trained positions
  auto pair_of = [&](double turns) { return rd * std::log(k.trained_len / (turns * two_pi)) / (2.0 * std::log(k.base)); };
  double lo = 0, hi = 0;
  if (k.scaling == INFS_ROTARY_YARN) {
    lo = std::max(std::floor(pair_of(k.high)), 0.0);
    hi = std::min(std::ceil(pair_of(k.low)), rd - 1.0);
  }
  for (int j = 0; j < r->pairs; ++j) {
    double f = std::pow(base, -2.0 * j / rd);
    if (k.scaling == INFS_ROTARY_LINEAR) {
      f /= s;
    } else if (k.scaling == INFS_ROTARY_YARN) {
      const double mix = std::min(1.0, std::max(0.0, (j - lo) / std::max(hi - lo, 0.001)));
      f = f / s * mix + f * (1.0 - mix);
    } else if (k.scaling == INFS_ROTARY_BANDS) {
      const double turns = k.trained_len * f / two_pi;
      const double mix = std::min(1.0, std::max(0.0, (turns - k.low) / (k.high - k.low)));
      f = (1.0 - mix) * f / s + mix * f;
    }
    r->freq[j] = f;
  }
  r->amplitude = k.amplitude > 0.0 ? k.amplitude : k.scaling == INFS_ROTARY_YARN ? 0.1 * std::log(s) + 1.0 : 1.0;
  *out = r;
  return INFS_OK;
}

void infs_rotary_destroy(infs_rotary* r) { delete r; }

infs_status infs_rotary_frequencies(const infs_rotary* r, double* freq_out, int32_t n, double* amplitude_out) {
  if (!r || !freq_out || !amplitude_out) return op_fail(INFS_E_ARG, "null argument");
  if (n != r->pairs) return op_fail(INFS_E_ARG, "n must equal rotary_dim / 2 = %d", r->pairs);
  std::copy(r->freq, r->freq + n, freq_out);
  *amplitude_out = r->amplitude;
  return INFS_OK;
}

infs_status infs_rotate_rows(const infs_rotary* r, void* hip_stream, int32_t dtype, int64_t tokens, const infs_rows* q,
                             const infs_rows* k, const int32_t* positions_dev, int32_t first_position, int32_t inverse) {
  if (!r) return op_fail(INFS_E_ARG, "null rotary configuration");
  if (dtype != INFS_F32 && dtype != INFS_BF16) return op_fail(INFS_E_ARG, "dtype must be INFS_F32 or INFS_BF16");
  if (tokens < 0 || tokens > INT32_MAX) return op_fail(INFS_E_ARG, "tokens must be in [0, 2^31)");
  if (!q && !k) return op_fail(INFS_E_ARG, "no rows given");
  if (!positions_dev && (int64_t)first_position + tokens - 1 > INT32_MAX)
    return op_fail(INFS_E_ARG, "positions beyond 2^31 - 1");
  if ((uintptr_t)positions_dev & 3) return op_fail(INFS_E_ARG, "positions must be aligned to 4 bytes");
  infs::RotaryArgs a{};
  infs_status st = INFS_OK;
  const size_t es = dtype == INFS_BF16 ? 2 : 4;
  const infs_rows* rows[2] = {q, k};
  for (int i = 0; i < 2 && st == INFS_OK; ++i) {
    if (!rows[i]) continue;
    st = infs::pack_rotary_rows(rows[i], i ? "k" : "q", r->cfg.head_dim, tokens, 1, es, i ? &a.k : &a.q);
    if (st == INFS_OK && tokens > 0 && (!rows[i]->in || !rows[i]->out)) st = op_fail(INFS_E_ARG, "null rows");
  }
  if (st != INFS_OK || tokens == 0) return st;
  infs::set_rotary(*r, inverse != 0, &a);
  a.positions = positions_dev;
  a.first = first_position;
  a.tokens = (int32_t)tokens;
  infs::StreamDevice dev((hipStream_t)hip_stream);
  hipError_t e = dev.status();
  if (e == hipSuccess)
    e = infs::launch_rotate(a, dtype == INFS_BF16, r->cfg.layout == INFS_ROTARY_INTERLEAVED, 1, (hipStream_t)hip_stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "rotating rows failed: %s", hipGetErrorString(e));
}

infs_status infs_scorer_create(const infs_scorer_config* cfg, void* hip_stream, infs_scorer** out) {
  if (!out) return op_fail(INFS_E_ARG, "out is null");
  *out = nullptr;
  if (!cfg) return op_fail(INFS_E_ARG, "cfg is null");
  const infs_scorer_config& k = *cfg;
  if (k.vocab < 1 || k.vocab > (1 << 24)) return op_fail(INFS_E_ARG, "vocab must be in [1, 2^24]");
  if (k.dtype != INFS_F32 && k.dtype != INFS_BF16) return op_fail(INFS_E_ARG, "dtype must be INFS_F32 or INFS_BF16");
  if (k.max_rows < 1 || k.max_rows > infs::kScoreMaxRows) return op_fail(INFS_E_ARG, "max_rows must be in [1, 2^23]");
  if (k.top_k < 0 || k.top_k > INFS_SCORE_MAX_TOP) return op_fail(INFS_E_ARG, "top_k must be in [0, %d]", INFS_SCORE_MAX_TOP);
  if (k.temperature != 0.f && !(k.temperature >= 0x1p-20f && k.temperature <= 0x1p20f))
    return op_fail(INFS_E_ARG, "temperature must be 0 (for 1) or in [2^-20, 2^20]");
  if (k.flags & ~INFS_FLAG_DRY_RUN) return op_fail(INFS_E_ARG, "unknown flags");
  infs_scorer* s = new (std::nothrow) infs_scorer;
  if (!s) return op_fail(INFS_E_NOMEM, "host allocation failed");
  s->cfg = k;
  s->dry = (k.flags & INFS_FLAG_DRY_RUN) != 0;
  s->bf16 = k.dtype == INFS_BF16;
  s->es = s->bf16 ? 2 : 4;
  s->inv_t = k.temperature != 0.f ? 1.f / k.temperature : 1.f;
  s->stream = (hipStream_t)hip_stream;
  if (!s->dry) {
    infs::StreamDevice dev(s->stream);
    hipError_t e = dev.status();
    if (e == hipSuccess) e = hipGetDevice(&s->device);
    if (e == hipSuccess) e = infs::score_resident(s->bf16, cfg->top_k > 0, &s->resident);
    if (e == hipSuccess) e = hipMalloc((void**)&s->workspace, workspace_bytes(*s));
    if (e == hipSuccess) e = hipMemset(s->workspace, 0, workspace_bytes(*s));
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);  // the stream need not wait for the null stream
    if (e != hipSuccess) {
      if (s->workspace) (void)hipFree(s->workspace);
      delete s;
      return op_fail(e == hipErrorOutOfMemory ? INFS_E_NOMEM : INFS_E_DEVICE, "a scorer's workspace: %s", hipGetErrorString(e));
    }
  }
  *out = s;
  return INFS_OK;
}

void infs_scorer_destroy(infs_scorer* s) {
  if (!s) return;
  if (!s->dry) {
    infs::StreamDevice dev(s->stream, s->device);
    (void)hipStreamSynchronize(s->stream);
    (void)hipFree(s->workspace);
  }
  delete s;
}

infs_status infs_score_tokens(infs_scorer* s, int32_t rows, const void* logits_dev, int64_t row_stride,
                              const int32_t* tokens_dev, float* logprob_dev, float* entropy_dev, int32_t* top_id_dev,
                              float* top_logprob_dev, float* stats_dev) {
  if (!s) return op_fail(INFS_E_ARG, "null scorer");
  const infs_status st = check_rows(s, rows, logits_dev, &row_stride, "logits");
  if (st != INFS_OK) return st;
  if (!tokens_dev != !logprob_dev) return op_fail(INFS_E_ARG, "tokens and logprob go together");
  if (!top_id_dev != !top_logprob_dev) return op_fail(INFS_E_ARG, "top_id and top_logprob go together");
  if (top_id_dev && s->cfg.top_k == 0) return op_fail(INFS_E_ARG, "alternatives need a scorer with top_k > 0");
  if (misaligned({tokens_dev, logprob_dev, entropy_dev, top_id_dev, top_logprob_dev}, 4) || misaligned({stats_dev}, 8))
    return op_fail(INFS_E_ARG, "tokens and outputs must be aligned to 4 bytes (stats: 8)");
  if (s->dry || rows == 0) return INFS_OK;
  infs::ScoreArgs a{logits_dev, row_stride, tokens_dev, logprob_dev, entropy_dev, top_id_dev, top_logprob_dev, stats_dev,
                    rows, s->cfg.vocab, top_id_dev ? s->cfg.top_k : 0, s->inv_t, 0, 0, 0,
                    s->resident, nullptr, nullptr, nullptr};
  char* ws = s->workspace;
  a.arrived = (int32_t*)ws;
  a.part = (float*)(ws + infs::kScoreArrivedBytes);
  a.keys = (unsigned long long*)(ws + infs::kScoreArrivedBytes + infs::kScorePartBytes);
  infs::StreamDevice dev(s->stream, s->device);
  hipError_t e = dev.status();
  if (e == hipSuccess) e = infs::launch_score(a, s->bf16, s->stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "scoring failed: %s", hipGetErrorString(e));
}

infs_status infs_score_grad(infs_scorer* s, int32_t rows, const void* logits_dev, int64_t row_stride,
                            const int32_t* tokens_dev, const float* stats_dev, const float* entropy_dev,
                            const float* d_logprob_dev, const float* d_entropy_dev, void* grad_dev,
                            int64_t grad_row_stride) {
  if (!s) return op_fail(INFS_E_ARG, "null scorer");
  infs_status st = check_rows(s, rows, logits_dev, &row_stride, "logits");
  if (st == INFS_OK) st = check_rows(s, rows, grad_dev, &grad_row_stride, "grad");
  if (st != INFS_OK) return st;
  if (d_logprob_dev && !tokens_dev) return op_fail(INFS_E_ARG, "d_logprob needs tokens");
  if (d_entropy_dev && !entropy_dev) return op_fail(INFS_E_ARG, "d_entropy needs entropy");
  if (rows > 0 && !s->dry && !stats_dev) return op_fail(INFS_E_ARG, "null stats");
  if (logits_dev && grad_dev == logits_dev && rows > 1 && row_stride != grad_row_stride)
    return op_fail(INFS_E_ARG, "a gradient over the logits needs their row stride");
  if (misaligned({tokens_dev, entropy_dev, d_logprob_dev, d_entropy_dev}, 4) || misaligned({stats_dev}, 8))
    return op_fail(INFS_E_ARG, "tokens and gradients must be aligned to 4 bytes (stats: 8)");
  if (s->dry || rows == 0) return INFS_OK;
  infs::ScoreGradArgs a{logits_dev, grad_dev, row_stride, grad_row_stride, d_logprob_dev ? tokens_dev : nullptr, stats_dev,
                        d_entropy_dev ? entropy_dev : nullptr, d_logprob_dev, d_entropy_dev, rows, s->cfg.vocab, s->inv_t, 0};
  infs::StreamDevice dev(s->stream, s->device);
  hipError_t e = dev.status();
  if (e == hipSuccess) e = infs::launch_score_grad(a, s->bf16, s->stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "the gradient of scores failed: %s", hipGetErrorString(e));
}

}  // extern "C"
