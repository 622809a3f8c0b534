// C ABI of the losses of sequences (see include/lvx.h): argument validation on the host and launches on the caller's stream.
#include "../../include/lvx.h"
#include "lvx_internal.h"

#include <cmath>

using namespace lvx;

namespace {

constexpr size_t ALIGN = 256;
size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
bool aligned(const void* p, size_t by) { return (uintptr_t)p % by == 0; }
bool sizes_ok(int64_t n, int64_t S) { return n >= 1 && S >= 1 && n <= (1 << 30) && S <= (1 << 21); }

size_t head_bytes(int64_t count) { return align_up(count * sequence_part_bytes()); }
size_t workspace_of(int64_t n, int64_t count) { return head_bytes(count) + align_up((n / SEQUENCE_BLOCK + 1) * sequence_part_bytes()); }

// what both have in common; `count`: sequences
lvx_status sequence_args(int64_t n, int64_t count, const float* nll, const float* ref, const int64_t* labels, const int64_t* first, float* loss,
                         const float* d_loss, float* d_nll, void* workspace, size_t workspace_bytes, SequenceArgs* a) {
  if (!nll || !labels || !first || !loss || (d_nll && !d_loss) || (d_loss && !d_nll)) return LVX_ERR_NULL;
  if (!aligned(nll, 4) || !aligned(ref, 4) || !aligned(labels, 8) || !aligned(first, 8) || !aligned(loss, 4) || !aligned(d_loss, 4) || !aligned(d_nll, 4))
    return LVX_ERR_STRIDE;
  if (!workspace || !aligned(workspace, ALIGN) || workspace_bytes < workspace_of(n, count)) return LVX_ERR_WORKSPACE;
  a->nll = nll; a->ref = ref; a->labels = labels; a->first = first; a->loss = loss; a->d_loss = d_loss; a->d_nll = d_nll;
  a->n = n; a->count = count;
  a->head = workspace;
  a->block = (char*)workspace + head_bytes(count);
  return LVX_OK;
}

}  // namespace

extern "C" {

size_t lvx_preference_workspace_bytes(int64_t n, int64_t S) { return sizes_ok(n, S) ? workspace_of(n, 2 * S) : 0; }

lvx_status lvx_preference(const lvx_pref* p, const float* nll, const float* ref, const int64_t* labels, const int64_t* first, float* loss,
                          float* margin, const float* d_loss, float* d_nll, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!p) return LVX_ERR_NULL;
  if (!sizes_ok(p->n, p->S)) return LVX_ERR_SHAPE;
  if (p->form < LVX_PREF_LOGISTIC || p->form > LVX_PREF_SQUARE) return LVX_ERR_UNSUPPORTED;
  if (!(p->beta > 0.0) || !std::isfinite(p->beta) || !(p->smoothing >= 0.0) || !(p->smoothing <= 1.0)) return LVX_ERR_SHAPE;
  if (p->smoothing != 0.0 && p->form != LVX_PREF_LOGISTIC) return LVX_ERR_UNSUPPORTED;
  SequenceArgs a{};
  const lvx_status st = sequence_args(p->n, 2 * p->S, nll, ref, labels, first, loss, d_loss, d_nll, workspace, workspace_bytes, &a);
  if (st != LVX_OK) return st;
  if (!aligned(margin, 4)) return LVX_ERR_STRIDE;
  // (a pair's d_loss is read by several workgroups, one of which writes its loss and margin)
  const int64_t len = p->S * 4, d = (int64_t)d_loss;
  if (d_loss && (rows_meet(d, 1, len, len, (int64_t)loss, len) || (margin && rows_meet(d, 1, len, len, (int64_t)margin, len)))) return LVX_ERR_STRIDE;
  a.margin = margin;
  a.form = p->form; a.beta = p->beta; a.smoothing = p->smoothing;
  return launch_preference(a, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

size_t lvx_policy_workspace_bytes(int64_t n, int64_t S) { return sizes_ok(n, S) ? workspace_of(n, S) : 0; }

lvx_status lvx_policy(const lvx_clip* p, const float* nll, const float* old, const float* ref, const float* adv, const int64_t* labels,
                      const int64_t* first, float* loss, float* stats, const float* d_loss, float* d_nll, void* workspace,
                      size_t workspace_bytes, void* hip_stream) {
  if (!p || !old || !adv) return LVX_ERR_NULL;
  if (!sizes_ok(p->n, p->S)) return LVX_ERR_SHAPE;
  for (const double x : {p->clip_low, p->clip_high, p->beta})
    if (!(x >= 0.0) || !std::isfinite(x)) return LVX_ERR_SHAPE;
  if (p->beta > 0.0 && !ref) return LVX_ERR_NULL;
  SequenceArgs a{};
  const lvx_status st = sequence_args(p->n, p->S, nll, ref, labels, first, loss, d_loss, d_nll, workspace, workspace_bytes, &a);
  if (st != LVX_OK) return st;
  if (!aligned(old, 4) || !aligned(adv, 4) || !aligned(stats, 4)) return LVX_ERR_STRIDE;
  a.old = old; a.adv = adv; a.stats = stats;
  a.mean = p->mean != 0; a.per_token = p->per_token != 0;
  a.beta = p->beta;
  a.low = 1.0 - p->clip_low; a.high = 1.0 + p->clip_high;
  a.ln_low = a.low > 0.0 ? std::log1p(-p->clip_low) : -HUGE_VAL;          // (a ratio is never below 0)
  a.ln_high = std::log1p(p->clip_high);
  return launch_policy(a, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

}  // extern "C"
