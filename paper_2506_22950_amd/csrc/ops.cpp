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

infs_status pack_norms(const infs_norms* n, NormWeights* out) {
  if (!n) return op_fail(INFS_E_ARG, "null norms");
  if (n->dtype != INFS_F32 && n->dtype != INFS_BF16) return op_fail(INFS_E_ARG, "norms: dtype must be INFS_F32 or INFS_BF16");
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return op_fail(INFS_E_ARG, "norms: eps must be finite and >= 0");
  if (n->layer_stride < 0 || n->layer_stride > (int64_t(1) << 40))
    return op_fail(INFS_E_ARG, "norms: layer_stride must be in [0, 2^40] elements");
  const size_t es = n->dtype == INFS_BF16 ? 2 : 4;
  if (((uintptr_t)n->weight_q | (uintptr_t)n->weight_k) % es)
    return op_fail(INFS_E_ARG, "norms: weights must be aligned to an element");
  out->weight[0] = n->weight_q;
  out->weight[1] = n->weight_k;
  out->weight_layer = n->layer_stride;
  out->eps = n->eps;
  out->weight_f32 = n->dtype == INFS_F32;
  return INFS_OK;
}

// Rows at positions: the checks of infs_rotate_rows and infs_norm_rotate_rows, and their launch arguments.
infs_status pack_rotation(const infs_rotary* r, int32_t dtype, int64_t tokens, const infs_rows* q, const infs_rows* k,
                          const int32_t* positions_dev, int32_t first_position, RotaryArgs* a) {
  if (!r) return op_fail(INFS_E_ARG, "null rotary configuration");
  if (dtype != INFS_F32 && dtype != INFS_BF16) return op_fail(INFS_E_ARG, "dtype must be INFS_F32 or INFS_BF16");
  if (tokens < 0 || tokens > INT32_MAX) return op_fail(INFS_E_ARG, "tokens must be in [0, 2^31)");
  if (!q && !k) return op_fail(INFS_E_ARG, "no rows given");
  if (!positions_dev && (int64_t)first_position + tokens - 1 > INT32_MAX)
    return op_fail(INFS_E_ARG, "positions beyond 2^31 - 1");
  if ((uintptr_t)positions_dev & 3) return op_fail(INFS_E_ARG, "positions must be aligned to 4 bytes");
  const size_t es = dtype == INFS_BF16 ? 2 : 4;
  const infs_rows* rows[2] = {q, k};
  for (int i = 0; i < 2; ++i) {
    if (!rows[i]) continue;
    const infs_status st = pack_rotary_rows(rows[i], i ? "k" : "q", r->cfg.head_dim, tokens, 1, es, i ? &a->k : &a->q);
    if (st != INFS_OK) return st;
    if (tokens > 0 && (!rows[i]->in || !rows[i]->out)) return op_fail(INFS_E_ARG, "null rows");
  }
  a->positions = positions_dev;
  a->first = first_position;
  a->tokens = (int32_t)tokens;
  return INFS_OK;
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

struct infs_sampler {
  infs_sampler_config cfg{};
  bool dry = false, bf16 = false;
  hipStream_t stream = nullptr;
  int device = 0;
  // Counters (zero before the first launch), states, lists and sums of rows and pieces (see ChooseArgs).
  char* workspace = nullptr;
  size_t list_n = 0, state = 0, list = 0, piece = 0, subs = 0, bins = 0;  // offsets
};

struct infs_attention {
  infs_attention_config cfg{};
  bool dry = false, bf16 = false;
  hipStream_t stream = nullptr;
  int device = 0;
  // [max_tokens, Hq] (AttendGradArgs), behind the parts of shared walks and their counters (AttendShape)
  float* delta = nullptr;
  float* part = nullptr;
  int32_t* arrived = nullptr;
};

namespace {

// Rows of an attention: E_ARG unless dense heads of whole 16-byte chunks; byte strides to row and head.
infs_status check_attend_rows(const infs_attention* a, const infs_rows* r, const char* what, int heads, int64_t tokens,
                              bool in, bool out, int64_t* in_row, int64_t* in_head, int64_t* out_row, int64_t* out_head) {
  if (!r) return op_fail(INFS_E_ARG, "%s: no rows given", what);
  if (r->heads != heads) return op_fail(INFS_E_ARG, "%s: %d heads, the attention has %d", what, r->heads, heads);
  infs_rows x = *r;
  if (!in) x.in = nullptr, x.in_row = x.in_head = 0;
  if (!out) x.out = nullptr, x.out_row = x.out_head = 0;
  x.in_layer = x.out_layer = 0;
  const int es = a->bf16 ? 2 : 4;
  if (in && out && x.in && x.in == x.out) return op_fail(INFS_E_ARG, "%s: outputs may not lie over the inputs", what);
  infs::RotaryRows p;
  const infs_status st = infs::pack_rotary_rows(&x, what, a->cfg.head_dim, tokens, 1, es, &p);
  if (st != INFS_OK) return st;
  if (!a->dry && tokens > 0 && ((in && !x.in) || (out && !x.out))) return op_fail(INFS_E_ARG, "%s: null rows", what);
  *in_row = p.in_row * es, *in_head = p.in_head * es;
  if (((uintptr_t)p.in | (uintptr_t)p.out | (uintptr_t)*in_row | (uintptr_t)*in_head | (uintptr_t)(p.out_row * es) |
       (uintptr_t)(p.out_head * es)) & 15)
    return op_fail(INFS_E_ARG, "%s: addresses and strides must be multiples of 16 bytes", what);
  if (out) *out_row = p.out_row * es, *out_head = p.out_head * es;
  return INFS_OK;
}

infs_status check_attend(const infs_attention* a, int32_t sequences, int64_t q_tokens, const int32_t* q_offsets,
                         int64_t* k_tokens, const int32_t** k_offsets, infs::AttendShape* s) {
  if (!a) return op_fail(INFS_E_ARG, "null attention");
  if (sequences < 0 || sequences > (1 << 20)) return op_fail(INFS_E_ARG, "sequences must be in [0, 2^20]");
  if (q_tokens < 0 || q_tokens > a->cfg.max_tokens)
    return op_fail(INFS_E_ARG, "q_tokens must be in [0, %d]", a->cfg.max_tokens);
  if (!*k_offsets) {
    if (*k_tokens != q_tokens) return op_fail(INFS_E_ARG, "without k_offsets the keys are the queries' tokens");
    *k_offsets = q_offsets;
  }
  if (*k_tokens < 0 || *k_tokens > INT32_MAX) return op_fail(INFS_E_ARG, "k_tokens must be in [0, 2^31)");
  if (((uintptr_t)q_offsets | (uintptr_t)*k_offsets) & 3) return op_fail(INFS_E_ARG, "offsets must be aligned to 4 bytes");
  if (!a->dry && sequences > 0 && !q_offsets) return op_fail(INFS_E_ARG, "null offsets");
  const int hpk = a->cfg.num_q_heads / a->cfg.num_kv_heads;
  // work-groups of the smallest tiles
  if ((q_tokens * hpk / 32 + sequences) * a->cfg.num_kv_heads > infs::kAttendMostBlocks ||
      (*k_tokens / 32 + sequences) * a->cfg.num_kv_heads > infs::kAttendMostBlocks)
    return op_fail(INFS_E_ARG, "more than 2^22 work-groups");
  *s = {q_offsets, *k_offsets, sequences, (int32_t)q_tokens, (int32_t)*k_tokens, a->cfg.num_q_heads, a->cfg.num_kv_heads, hpk,
        (uint32_t)(((uint64_t(1) << 32) + hpk - 1) / hpk), a->cfg.scale, a->part, a->arrived, 1, 0};
  return INFS_OK;
}

infs_status check_rows(const infs_scorer* s, int32_t rows, const void* logits, int64_t* stride, const char* what) {
  if (rows < 0 || rows > s->cfg.max_rows) return op_fail(INFS_E_ARG, "rows must be in [0, %d]", s->cfg.max_rows);
  if (*stride == 0) *stride = s->cfg.vocab;
  if (*stride < s->cfg.vocab || *stride > (int64_t(1) << 40))
    return op_fail(INFS_E_ARG, "%s: row stride must be 0 or in [vocab, 2^40]", what);
  if (rows > 0 && !s->dry && !logits) return op_fail(INFS_E_ARG, "%s: null buffer", what);
  if ((uintptr_t)logits % s->es) return op_fail(INFS_E_ARG, "%s must be aligned to an element", what);
  return INFS_OK;
}

// Lays out a sampler's workspace for its largest call; returns its bytes.
size_t lay_out(infs_sampler* s) {
  int64_t rows = 0, pieces = 0;  // of one launch
  const auto call = [&](int n) {
    const int p = infs::choose_pieces(s->cfg.vocab, infs::choose_batches(n, s->cfg.vocab, s->bf16), s->bf16);
    const int64_t r = std::min(n, infs::choose_rows(p));
    rows = std::max(rows, r);
    pieces = std::max(pieces, r * p);
  };
  for (int n = 1; n <= std::min(s->cfg.max_rows, infs::kChooseRows); ++n) call(n);
  call(s->cfg.max_rows);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t begin = at;
    at += (bytes + 255) / 256 * 256;
    return begin;
  };
  take(sizeof(int32_t) * infs::kCounterStride * rows);
  s->list_n = take(sizeof(int32_t) * infs::kCounterStride * rows);
  s->state = take(sizeof(infs::RowState) * rows);
  s->list = take(sizeof(unsigned long long) * infs::kList * rows);
  s->piece = take(sizeof(infs::PieceState) * pieces);
  s->subs = take(sizeof(unsigned long long) * infs::kChooseSubs * pieces);
  s->bins = take(sizeof(uint32_t) * infs::kBins * pieces);
  return at;
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
  infs::RotaryArgs a{};
  const infs_status st = infs::pack_rotation(r, dtype, tokens, q, k, positions_dev, first_position, &a);
  if (st != INFS_OK || tokens == 0) return st;
  infs::set_rotary(*r, inverse != 0, &a);
  infs::StreamDevice dev((hipStream_t)hip_stream);
  hipError_t e = dev.status();
  if (e == hipSuccess)
    e = infs::launch_rotate(a, dtype == INFS_BF16, r->cfg.layout == INFS_ROTARY_INTERLEAVED, 1, (hipStream_t)hip_stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "rotating rows failed: %s", hipGetErrorString(e));
}

infs_status infs_norm_rotate_rows(const infs_rotary* r, void* hip_stream, int32_t dtype, int64_t tokens,
                                  const infs_norms* norms, const infs_rows* q, const infs_rows* k,
                                  const int32_t* positions_dev, int32_t first_position) {
  infs::NormArgs a{};
  infs_status st = infs::pack_rotation(r, dtype, tokens, q, k, positions_dev, first_position, &a.r);
  if (st == INFS_OK) st = infs::pack_norms(norms, &a);
  if (st != INFS_OK || tokens == 0) return st;
  infs::set_rotary(*r, false, &a.r);
  infs::StreamDevice dev((hipStream_t)hip_stream);
  hipError_t e = dev.status();
  if (e == hipSuccess)
    e = infs::launch_norm_rotate(a, dtype == INFS_BF16, r->cfg.layout == INFS_ROTARY_INTERLEAVED, 1, (hipStream_t)hip_stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "norms of rows failed: %s", hipGetErrorString(e));
}

int64_t infs_norm_rotate_grad_workspace(int64_t tokens, int32_t head_dim) {
  if (tokens <= 0 || head_dim <= 0) return 0;
  return (int64_t)sizeof(float) * 2 * infs::norm_grad_parts(tokens) * head_dim;
}

infs_status infs_norm_rotate_grad(const infs_rotary* r, void* hip_stream, int32_t dtype, int64_t tokens,
                                  const infs_norms* norms, const infs_rows* q, const infs_rows* k, const infs_rows* dq,
                                  const infs_rows* dk, float* d_weight_q_dev, float* d_weight_k_dev, void* workspace_dev,
                                  const int32_t* positions_dev, int32_t first_position) {
  infs::NormGradArgs a{};
  infs_status st = infs::pack_rotation(r, dtype, tokens, q, k, positions_dev, first_position, &a.r);
  if (st == INFS_OK) st = infs::pack_norms(norms, &a);
  if (st != INFS_OK) return st;
  if (!q != !dq || !k != !dk) return op_fail(INFS_E_ARG, "q and dq go together, and k and dk");
  const infs_rows* rows[2] = {q, k};
  const infs_rows* grads[2] = {dq, dk};
  for (int i = 0; i < 2; ++i) {
    if (!grads[i]) continue;
    const char* what = i ? "dk" : "dq";
    if (grads[i]->heads != rows[i]->heads) return op_fail(INFS_E_ARG, "%s: as many heads as the rows", what);
    infs_rows g = *grads[i];  // written over: by the strides of the rows' gradients
    g.out = g.in == rows[i]->out ? rows[i]->out : nullptr;
    g.out_row = rows[i]->out_row, g.out_head = rows[i]->out_head, g.out_layer = 0, g.in_layer = 0;
    st = infs::pack_rotary_rows(&g, what, r->cfg.head_dim, tokens, 1, dtype == INFS_BF16 ? 2 : 4, i ? &a.dk : &a.dq);
    if (st != INFS_OK) return st;
    if (tokens > 0 && !g.in) return op_fail(INFS_E_ARG, "%s: null rows", what);
  }
  if ((d_weight_q_dev && !q) || (d_weight_k_dev && !k)) return op_fail(INFS_E_ARG, "a gradient of weights without rows");
  if (((uintptr_t)d_weight_q_dev | (uintptr_t)d_weight_k_dev) & 3)
    return op_fail(INFS_E_ARG, "gradients of weights must be aligned to 4 bytes");
  if ((uintptr_t)workspace_dev & 15) return op_fail(INFS_E_ARG, "the workspace must be aligned to 16 bytes");
  if (tokens > 0 && (d_weight_q_dev || d_weight_k_dev) && !workspace_dev)
    return op_fail(INFS_E_ARG, "gradients of weights need a workspace");
  infs::set_rotary(*r, false, &a.r);
  a.sums[0] = d_weight_q_dev;
  a.sums[1] = d_weight_k_dev;
  a.part = (float*)workspace_dev;
  infs::StreamDevice dev((hipStream_t)hip_stream);
  hipError_t e = dev.status();
  if (e == hipSuccess)
    e = infs::launch_norm_rotate_grad(a, dtype == INFS_BF16, r->cfg.layout == INFS_ROTARY_INTERLEAVED, (hipStream_t)hip_stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "the gradient of norms failed: %s", hipGetErrorString(e));
}

infs_status infs_attention_create(const infs_attention_config* cfg, void* hip_stream, infs_attention** out) {
  if (!out) return op_fail(INFS_E_ARG, "out is null");
  *out = nullptr;
  if (!cfg) return op_fail(INFS_E_ARG, "cfg is null");
  const infs_attention_config& k = *cfg;
  if (k.num_kv_heads < 1 || k.num_q_heads < 1 || k.num_q_heads > 4096 || k.num_q_heads % k.num_kv_heads)
    return op_fail(INFS_E_ARG, "num_q_heads must be a multiple of num_kv_heads, up to 4096");
  if (k.head_dim != 64 && k.head_dim != 128) return op_fail(INFS_E_ARG, "head_dim must be 64 or 128");
  if (k.dtype != INFS_F32 && k.dtype != INFS_BF16) return op_fail(INFS_E_ARG, "dtype must be INFS_F32 or INFS_BF16");
  if (k.scale != 0.f && !(k.scale >= 0x1p-64f && k.scale <= 0x1p64f))
    return op_fail(INFS_E_ARG, "scale must be in [2^-64, 2^64], or 0");
  if (k.max_tokens < 1 || (int64_t)k.max_tokens * (k.num_q_heads / k.num_kv_heads) > INT32_MAX)
    return op_fail(INFS_E_ARG, "max_tokens must be at least 1, times Hq / Hkv below 2^31");
  if (k.flags & ~INFS_FLAG_DRY_RUN) return op_fail(INFS_E_ARG, "unknown flags");
  infs_attention* a = new (std::nothrow) infs_attention;
  if (!a) return op_fail(INFS_E_NOMEM, "host allocation failed");
  a->cfg = k;
  if (k.scale == 0.f) a->cfg.scale = 1.f / std::sqrt((float)k.head_dim);
  a->dry = (k.flags & INFS_FLAG_DRY_RUN) != 0;
  a->bf16 = k.dtype == INFS_BF16;
  a->stream = (hipStream_t)hip_stream;
  if (!a->dry) {
    infs::StreamDevice dev(a->stream);
    hipError_t e = dev.status();
    if (e == hipSuccess) e = hipGetDevice(&a->device);
    const size_t counters = sizeof(int32_t) * infs::kAttendParts,
                 parts = sizeof(float) * infs::kAttendParts * infs::kAttendPartFloats * k.head_dim,
                 delta = sizeof(float) * k.max_tokens * k.num_q_heads;
    char* all = nullptr;
    if (e == hipSuccess) e = hipMalloc((void**)&all, counters + parts + delta);
    if (e == hipSuccess) {
      a->arrived = (int32_t*)all, a->part = (float*)(all + counters), a->delta = (float*)(all + counters + parts);
      e = hipMemset(a->arrived, 0, counters);
      if (e == hipSuccess) e = hipStreamSynchronize(nullptr);  // the stream need not wait for the null stream
    }
    if (e != hipSuccess) {
      if (all) (void)hipFree(all);
      delete a;
      return op_fail(e == hipErrorOutOfMemory ? INFS_E_NOMEM : INFS_E_DEVICE, "an attention's workspace: %s",
                     hipGetErrorString(e));
    }
  }
  *out = a;
  return INFS_OK;
}

void infs_attention_destroy(infs_attention* a) {
  if (!a) return;
  if (!a->dry) {
    infs::StreamDevice dev(a->stream, a->device);
    (void)hipStreamSynchronize(a->stream);
    (void)hipFree(a->arrived);
  }
  delete a;
}

infs_status infs_attend(infs_attention* a, int32_t sequences, int64_t q_tokens, const int32_t* q_offsets_dev,
                        int64_t k_tokens, const int32_t* k_offsets_dev, const infs_rows* q, const infs_rows* k,
                        const infs_rows* v, float* lse_dev) {
  infs::AttendArgs x{};
  infs_status st = check_attend(a, sequences, q_tokens, q_offsets_dev, &k_tokens, &k_offsets_dev, &x);
  if (st != INFS_OK) return st;
  const int hq = a->cfg.num_q_heads, hkv = a->cfg.num_kv_heads;
  st = check_attend_rows(a, q, "q", hq, q_tokens, true, true, &x.q_row, &x.q_head, &x.o_row, &x.o_head);
  if (st == INFS_OK) st = check_attend_rows(a, k, "k", hkv, k_tokens, true, false, &x.k_row, &x.k_head, nullptr, nullptr);
  if (st == INFS_OK) st = check_attend_rows(a, v, "v", hkv, k_tokens, true, false, &x.v_row, &x.v_head, nullptr, nullptr);
  if (st != INFS_OK) return st;
  if ((uintptr_t)lse_dev & 3) return op_fail(INFS_E_ARG, "lse must be aligned to 4 bytes");
  if (a->dry || sequences == 0 || q_tokens == 0) return INFS_OK;
  x.q = (const char*)q->in, x.k = (const char*)k->in, x.v = (const char*)v->in, x.o = (char*)q->out;
  x.lse = lse_dev;
  infs::StreamDevice dev(a->stream, a->device);
  hipError_t e = dev.status();
  if (e == hipSuccess) e = infs::launch_attend(x, a->bf16, a->cfg.head_dim, a->stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "attention failed: %s", hipGetErrorString(e));
}

infs_status infs_attend_grad(infs_attention* a, int32_t sequences, int64_t q_tokens, const int32_t* q_offsets_dev,
                             int64_t k_tokens, const int32_t* k_offsets_dev, const infs_rows* q, const infs_rows* k,
                             const infs_rows* v, const infs_rows* o, const infs_rows* d_o, const float* lse_dev) {
  infs::AttendGradArgs x{};
  infs_status st = check_attend(a, sequences, q_tokens, q_offsets_dev, &k_tokens, &k_offsets_dev, &x);
  if (st != INFS_OK) return st;
  const int hq = a->cfg.num_q_heads, hkv = a->cfg.num_kv_heads;
  st = check_attend_rows(a, q, "q", hq, q_tokens, true, true, &x.q_row, &x.q_head, &x.dq_row, &x.dq_head);
  if (st == INFS_OK) st = check_attend_rows(a, k, "k", hkv, k_tokens, true, true, &x.k_row, &x.k_head, &x.dk_row, &x.dk_head);
  if (st == INFS_OK) st = check_attend_rows(a, v, "v", hkv, k_tokens, true, true, &x.v_row, &x.v_head, &x.dv_row, &x.dv_head);
  if (st == INFS_OK) st = check_attend_rows(a, o, "o", hq, q_tokens, true, false, &x.o_row, &x.o_head, nullptr, nullptr);
  if (st == INFS_OK) st = check_attend_rows(a, d_o, "d_o", hq, q_tokens, true, false, &x.do_row, &x.do_head, nullptr, nullptr);
  if (st != INFS_OK) return st;
  if ((uintptr_t)lse_dev & 3) return op_fail(INFS_E_ARG, "lse must be aligned to 4 bytes");
  if (!a->dry && q_tokens > 0 && !lse_dev) return op_fail(INFS_E_ARG, "null lse");
  if (a->dry || sequences == 0) return INFS_OK;
  x.q = (const char*)q->in, x.k = (const char*)k->in, x.v = (const char*)v->in, x.o = (const char*)o->in;
  x.d_o = (const char*)d_o->in, x.dq = (char*)q->out, x.dk = (char*)k->out, x.dv = (char*)v->out;
  x.lse = lse_dev;
  x.delta = a->delta;
  infs::StreamDevice dev(a->stream, a->device);
  hipError_t e = dev.status();
  if (e == hipSuccess) e = infs::launch_attend_grad(x, a->bf16, a->cfg.head_dim, a->stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "the gradient of attention failed: %s", hipGetErrorString(e));
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

infs_status infs_sampler_create(const infs_sampler_config* cfg, void* hip_stream, infs_sampler** out) {
  if (!out) return op_fail(INFS_E_ARG, "out is null");
  *out = nullptr;
  if (!cfg) return op_fail(INFS_E_ARG, "cfg is null");
  const infs_sampler_config& k = *cfg;
  if (k.vocab < 1 || k.vocab > (1 << 24)) return op_fail(INFS_E_ARG, "vocab must be in [1, 2^24]");
  if (k.dtype != INFS_F32 && k.dtype != INFS_BF16) return op_fail(INFS_E_ARG, "dtype must be INFS_F32 or INFS_BF16");
  if (k.max_rows < 1 || k.max_rows > infs::kChooseMaxRows) return op_fail(INFS_E_ARG, "max_rows must be in [1, 2^22]");
  if (k.flags & ~INFS_FLAG_DRY_RUN) return op_fail(INFS_E_ARG, "unknown flags");
  infs_sampler* s = new (std::nothrow) infs_sampler;
  if (!s) return op_fail(INFS_E_NOMEM, "host allocation failed");
  s->cfg = k;
  s->dry = (k.flags & INFS_FLAG_DRY_RUN) != 0;
  s->bf16 = k.dtype == INFS_BF16;
  s->stream = (hipStream_t)hip_stream;
  if (!s->dry) {
    infs::StreamDevice dev(s->stream);
    hipError_t e = dev.status();
    if (e == hipSuccess) e = hipGetDevice(&s->device);
    const size_t bytes = lay_out(s);
    if (e == hipSuccess) e = hipMalloc((void**)&s->workspace, bytes);
    if (e == hipSuccess) e = hipMemset(s->workspace, 0, s->state);  // the counters
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);  // the stream need not wait for the null stream
    if (e != hipSuccess) {
      if (s->workspace) (void)hipFree(s->workspace);
      delete s;
      return op_fail(e == hipErrorOutOfMemory ? INFS_E_NOMEM : INFS_E_DEVICE, "a sampler's workspace: %s", hipGetErrorString(e));
    }
  }
  *out = s;
  return INFS_OK;
}

void infs_sampler_destroy(infs_sampler* s) {
  if (!s) return;
  if (!s->dry) {
    infs::StreamDevice dev(s->stream, s->device);
    (void)hipStreamSynchronize(s->stream);
    (void)hipFree(s->workspace);
  }
  delete s;
}

infs_status infs_choose_tokens(infs_sampler* s, int32_t rows, const void* logits_dev, int64_t row_stride,
                               const float* uniform_dev, const infs_sampling* all, const infs_sampling* each_dev,
                               int32_t* token_dev, float* logprob_dev, int32_t* kept_dev) {
  if (!s) return op_fail(INFS_E_ARG, "null sampler");
  if (rows < 0 || rows > s->cfg.max_rows) return op_fail(INFS_E_ARG, "rows must be in [0, %d]", s->cfg.max_rows);
  if (row_stride == 0) row_stride = s->cfg.vocab;
  if (row_stride < s->cfg.vocab || row_stride > (int64_t(1) << 40))
    return op_fail(INFS_E_ARG, "row stride must be 0 or in [vocab, 2^40]");
  if (rows > 0 && !s->dry && (!logits_dev || !uniform_dev || !token_dev)) return op_fail(INFS_E_ARG, "null buffer");
  if ((uintptr_t)logits_dev % (s->bf16 ? 2 : 4)) return op_fail(INFS_E_ARG, "logits must be aligned to an element");
  if (misaligned({uniform_dev, token_dev, logprob_dev, kept_dev}, 4) || misaligned({each_dev}, 8))
    return op_fail(INFS_E_ARG, "uniform numbers and outputs must be aligned to 4 bytes (each: 8)");
  const infs_sampling none{}, &p = all ? *all : none;
  if (!each_dev) {
    if (p.temperature != 0.0 && !(p.temperature >= 0x1p-20 && p.temperature <= 0x1p20))
      return op_fail(INFS_E_ARG, "temperature must be 0 (for 1) or in [2^-20, 2^20]");
    if (!(p.top_p >= 0.0 && p.top_p <= 1.0)) return op_fail(INFS_E_ARG, "top_p must be 0 (for 1) or in (0, 1]");
    if (!(p.min_p >= 0.0 && p.min_p <= 1.0)) return op_fail(INFS_E_ARG, "min_p must be in [0, 1]");
    if (p.top_k < 0) return op_fail(INFS_E_ARG, "top_k must be >= 0");
    if (p.reserved != 0) return op_fail(INFS_E_ARG, "reserved must be 0");
  }
  if (s->dry || rows == 0) return INFS_OK;
  infs::ChooseArgs a{logits_dev, row_stride, uniform_dev, each_dev, p, token_dev, logprob_dev, kept_dev, rows, s->cfg.vocab};
  char* ws = s->workspace;
  a.arrived = (int32_t*)ws;
  a.list_n = (int32_t*)(ws + s->list_n);
  a.state = (infs::RowState*)(ws + s->state);
  a.list = (unsigned long long*)(ws + s->list);
  a.piece = (infs::PieceState*)(ws + s->piece);
  a.subs = (unsigned long long*)(ws + s->subs);
  a.bins = (uint32_t*)(ws + s->bins);
  infs::StreamDevice dev(s->stream, s->device);
  hipError_t e = dev.status();
  if (e == hipSuccess) e = infs::launch_choose(a, s->bf16, s->stream);
  return e == hipSuccess ? INFS_OK : op_fail(INFS_E_DEVICE, "choosing tokens failed: %s", hipGetErrorString(e));
}

}  // extern "C"
