// C ABI of the losses against a vocabulary, cross entropy and distillation (see include/lvx.h): argument validation on the host, workspace carving, and
// launches on the caller's stream.
#include "../../include/lvx.h"
#include "lvx_internal.h"

using namespace lvx;

namespace {

constexpr size_t ALIGN = 256;
size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
bool aligned(const void* p, size_t by) { return (uintptr_t)p % by == 0; }

// Whether dx or dw lies in x or w, or one in the other (windows of one wider tensor beside each other do not)
bool gradients_in_operands(const lvx_xent* p, int64_t el, const void* x, const void* w, const void* dx, const void* dw) {
  const int64_t pitch = p->x_ss * el, row = p->E * el, vocab = p->V * row, xa = (int64_t)x, wa = (int64_t)w, dxa = (int64_t)dx, dwa = (int64_t)dw;
  return (dx && (rows_meet(xa - (p->n - 1) * pitch, 2 * p->n - 1, pitch, row, dxa, row) || rows_meet(dxa, p->n, pitch, row, wa, vocab))) ||
         (dw && (rows_meet(wa, 1, vocab, vocab, dwa, vocab) || rows_meet(xa, p->n, pitch, row, dwa, vocab))) ||
         (dx && dw && rows_meet(dxa, p->n, pitch, row, dwa, vocab));
}

lvx_status check_sizes(int64_t n, int32_t E, int64_t V, lvx_dtype dtype) {
  if (dtype != LVX_F32 && dtype != LVX_BF16) return LVX_ERR_DTYPE;
  if (n < 1 || E < 1 || V < 1 || n > (1 << 30) || V > (1 << 30) || E > (1 << 20)) return LVX_ERR_SHAPE;
  if (dtype == LVX_BF16 && !xent_bf16_supported(E)) return LVX_ERR_UNSUPPORTED;
  return LVX_OK;
}

// The workspace: the list of tokens; then (forward) what the tiles leave, or (backward) dx's sums, the gradient of a piece of the logits
// and dw's sums.
struct Plan { size_t tok, lab, zlab, part, fwd, dx, g, row; int64_t Mp, slots; };
Plan plan_of(int64_t n, int32_t E, int64_t V, lvx_dtype dtype) {
  const int f32 = dtype == LVX_F32;
  Plan p;
  p.slots = xent_dx_slots(n, E, V, device_cu_count(), f32);
  p.Mp = (n + 255) / 256 * 256;
  p.tok = ALIGN;
  p.lab = p.tok + align_up(n * 4);
  p.zlab = p.lab + align_up(n * 4);
  p.part = p.dx = p.zlab + align_up(n * 8);              // (zlab: the forward pass's label logits or the backward pass's rows)
  p.fwd = p.part + (size_t)xent_stat_parts(V, f32) * p.Mp * sizeof(float2);
  p.g = p.dx + align_up(xent_dx_bytes(n, E, V, device_cu_count(), f32));
  p.row = (size_t)p.Mp * (f32 ? 4 : 2);                // bytes of a column of the logits' gradient
  return p;
}
// Columns between the rows of the logits' gradient that nobody fills: a power of two from row to row would put a column's lines into few of the
// memory's channels (1000 x 2048 against 16384, dx: 66 -> 60 us).
constexpr int64_t PAD = 64;
// Columns of a piece of the vocabulary: a GiB of the logits' gradient, 8192 at least, since the sums of dx go through memory once a
// piece.  Pieces that the last-level cache (256 MB) holds gain nothing, and more of them have more last rounds of workgroups: passes with 128 MB,
// 512 MB and 1 GiB, us, in one session: 5514 x 1024, V = 50021, 2200 labelled 1088, 999, 966; 16000 x 1024, V = 32000 4710, 4180, 3750;
// 4096 x 4096, V = 131072 13880, 13840, 13790.
constexpr size_t PIECE_BYTES = (size_t)1 << 30;
constexpr int64_t LEAST_PIECE = 8192, MOST_PIECE = 1 << 18;
int64_t piece_of(const Plan& p, int64_t V) {
  int64_t piece = (int64_t)(PIECE_BYTES / p.row) / 256 * 256;
  if (piece < LEAST_PIECE) piece = LEAST_PIECE;
  if (piece > MOST_PIECE) piece = MOST_PIECE;
  const int64_t pieces = (V + piece - 1) / piece;      // (even ones)
  return ((V + pieces - 1) / pieces + 255) / 256 * 256;
}
// Room for a piece, and for a piece of every problem with fewer tokens or entries: even pieces get shorter where one more begins, and those of
// fewer tokens longer, so theirs may be the larger ones.
size_t piece_room(const Plan& p, int64_t V) {
  size_t room = p.row * LEAST_PIECE;
  if (room < PIECE_BYTES) room = PIECE_BYTES;
  if (room > p.row * MOST_PIECE) room = p.row * MOST_PIECE;
  const size_t all = p.row * ((V + 255) / 256 * 256);
  return (room < all ? room : all) + p.row * PAD;
}

lvx_status xent_args(const lvx_xent* p, lvx_dtype dtype, const void* x, const void* w, const int64_t* labels, void* workspace,
                     XentArgs* a, Plan* plan) {
  if (!p || !x || !w || !labels) return LVX_ERR_NULL;
  const lvx_status st = check_sizes(p->n, p->E, p->V, dtype);
  if (st != LVX_OK) return st;
  const size_t el = dtype == LVX_F32 ? 4 : 2;
  if (p->x_ss < p->E || p->n * (double)p->x_ss > 2147483648.0) return LVX_ERR_STRIDE;
  if (dtype == LVX_BF16 ? !aligned(x, 16) || !aligned(w, 16) || p->x_ss % 8 != 0 : !aligned(x, el) || !aligned(w, el)) return LVX_ERR_STRIDE;
  if (!aligned(labels, 8)) return LVX_ERR_STRIDE;
  if (!workspace || !aligned(workspace, ALIGN)) return LVX_ERR_WORKSPACE;
  *plan = plan_of(p->n, p->E, p->V, dtype);
  *a = XentArgs{};
  a->x = x; a->w = w; a->labels = labels;
  a->n = p->n; a->ldx = p->x_ss; a->V = p->V; a->E = p->E; a->n_cu = device_cu_count();
  const auto at = [&](size_t o) -> char* { return (char*)workspace + o; };
  a->head = (XentHead*)workspace;
  a->tok = (int*)at(plan->tok); a->lab = (int*)at(plan->lab); a->zlab = (float*)at(plan->zlab); a->row = (float2*)at(plan->zlab);
  a->part = (float2*)at(plan->part); a->dx_part = (float*)at(plan->dx); a->g = at(plan->g);
  a->Mp = plan->Mp;
  a->slots = (int)plan->slots;
  a->inv_t = 1.f;
  return LVX_OK;
}
// ... and of the backward pass
lvx_status xent_bwd_args(const lvx_xent* p, lvx_dtype dtype, const void* x, const void* w, const int64_t* labels, const float* lse,
                         const float* d_loss, void* dx, void* dw, void* workspace, size_t workspace_bytes, XentArgs* a) {
  Plan plan;
  if (!lse || !d_loss || (!dx && !dw)) return LVX_ERR_NULL;
  const lvx_status st = xent_args(p, dtype, x, w, labels, workspace, a, &plan);
  if (st != LVX_OK) return st;
  const size_t out = dtype == LVX_F32 ? 4 : 16;
  if (!aligned(lse, 4) || !aligned(d_loss, 4) || !aligned(dx, out) || !aligned(dw, out) || dx == x) return LVX_ERR_STRIDE;
  // the piece that there is room for
  int64_t piece = piece_of(plan, p->V);
  const int64_t room = workspace_bytes > plan.g ? ((int64_t)((workspace_bytes - plan.g) / plan.row) - PAD) / 256 * 256 : 0;
  if (piece > room) piece = room;
  if (piece < 256) return LVX_ERR_WORKSPACE;
  if (gradients_in_operands(p, dtype == LVX_F32 ? 4 : 2, x, w, dx, dw)) return LVX_ERR_STRIDE;
  a->piece = piece;
  a->g_pitch = piece + PAD;
  a->lse = lse; a->d_loss = d_loss; a->dx = dx; a->dw = dw;
  // parts of dw, if there is room for them behind it
  const int64_t cols = piece < p->V ? piece : p->V;
  const size_t end = align_up(plan.g + (size_t)a->g_pitch * plan.row);
  if (end + xent_dw_bytes(p->n, p->E, cols, a->n_cu, dtype == LVX_F32) <= workspace_bytes) {
    a->dw_slots = (int)xent_dw_slots(p->n, p->E, cols, a->n_cu, dtype == LVX_F32);
    a->dw_part = (float*)((char*)workspace + end);
  }
  return LVX_OK;
}

// Distillation: in front of the workspace of the cross entropy, what the tokens' entries need (backward: the first two of it)
struct EntryPlan { size_t q_stat, sorted, rank, starts, z, fwd, bwd; };
EntryPlan entries_of(int64_t n, int64_t V, int32_t K) {
  EntryPlan e;
  size_t at = align_up(n * 8);                       // (labels)
  e.q_stat = at; at += align_up(n * 8);
  e.bwd = at;
  e.sorted = at; at += align_up((size_t)n * K * 4 + 16);      // (they are read four at a time)
  e.rank = at; at += align_up((size_t)n * K * 2);
  e.starts = at; at += align_up((size_t)n * ((V + 63) / 64 + 1) * 2);
  e.z = at; at += align_up((size_t)n * K * 4);
  e.fwd = at;
  return e;
}
float log2_over(float temperature) { return (float)(1.4426950408889634 / temperature); }      // log2 e / temperature
bool entries_ok(int32_t K) { return K >= 1 && K <= DISTIL_MOST_ENTRIES; }
// what a call names beside the product's operands
lvx_status distil_check(const lvx_distil* p, lvx_dtype dtype, const int64_t* ids, const void* teacher, lvx_dtype teacher_dtype, const void* loss,
                        const void* lse, const void* ln_p, const void* workspace) {
  if (!p || !ids || !teacher || !loss || !lse || !ln_p) return LVX_ERR_NULL;
  const lvx_status st = check_sizes(p->n, p->E, p->V, dtype);
  if (st != LVX_OK) return st;
  if (teacher_dtype != LVX_F32 && teacher_dtype != LVX_BF16) return LVX_ERR_DTYPE;
  if (p->K < 1) return LVX_ERR_SHAPE;
  if (!entries_ok(p->K)) return LVX_ERR_UNSUPPORTED;
  if (!(p->temperature > 0.f) || !(1.f / p->temperature > 0.f) || !(log2_over(p->temperature) < __builtin_inff())) return LVX_ERR_SHAPE;
  if (!aligned(ids, 8) || !aligned(teacher, teacher_dtype == LVX_F32 ? 4 : 2) || !aligned(loss, 4) || !aligned(lse, 4) || !aligned(ln_p, 4))
    return LVX_ERR_STRIDE;
  return workspace && aligned(workspace, ALIGN) ? LVX_OK : LVX_ERR_WORKSPACE;
}
void distil_args(const lvx_distil* p, const int64_t* ids, const void* teacher, lvx_dtype teacher_dtype, float* ln_p, void* workspace, XentArgs* a) {
  const EntryPlan e = entries_of(p->n, p->V, p->K);
  const auto at = [&](size_t o) -> char* { return (char*)workspace + o; };
  a->temperature = p->temperature;
  a->inv_t = 1.f / p->temperature;
  a->z2 = log2_over(p->temperature);
  a->K = p->K;
  a->blocks = (int)((p->V + 63) / 64);
  a->ids = ids; a->teacher = teacher; a->teacher_bf16 = teacher_dtype == LVX_BF16; a->ln_p = ln_p;
  a->q_stat = (float2*)at(e.q_stat); a->sorted = (int*)at(e.sorted); a->rank = (uint16_t*)at(e.rank); a->starts = (uint16_t*)at(e.starts);
  a->z_entry = (float*)at(e.z);
}

}  // namespace

extern "C" {

size_t lvx_xent_workspace_bytes(int64_t n, int32_t E, int64_t V, lvx_dtype dtype) {
  if (check_sizes(n, E, V, dtype) != LVX_OK) return 0;
  const Plan p = plan_of(n, E, V, dtype);
  const size_t bwd = align_up(p.g + piece_room(p, V)) + xent_dw_room(n, E, V, device_cu_count(), dtype == LVX_F32);
  return align_up(p.fwd > bwd ? p.fwd : bwd);
}

lvx_status lvx_xent_fwd(const lvx_xent* p, lvx_dtype dtype, const void* x, const void* w, const int64_t* labels, float* loss, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  XentArgs a;
  Plan plan;
  if (!loss || !lse) return LVX_ERR_NULL;
  const lvx_status st = xent_args(p, dtype, x, w, labels, workspace, &a, &plan);
  if (st != LVX_OK) return st;
  if (!aligned(loss, 4) || !aligned(lse, 4)) return LVX_ERR_STRIDE;
  if (workspace_bytes < plan.fwd) return LVX_ERR_WORKSPACE;
  a.loss = loss; a.lse_out = lse;
  return launch_xent_fwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

lvx_status lvx_xent_bwd(const lvx_xent* p, lvx_dtype dtype, const void* x, const void* w, const int64_t* labels, const float* lse,
                        const float* d_loss, void* dx, void* dw, void* workspace, size_t workspace_bytes, void* hip_stream) {
  XentArgs a;
  const lvx_status st = xent_bwd_args(p, dtype, x, w, labels, lse, d_loss, dx, dw, workspace, workspace_bytes, &a);
  if (st != LVX_OK) return st;
  return launch_xent_bwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

size_t lvx_distil_workspace_bytes(int64_t n, int32_t E, int64_t V, int32_t K, lvx_dtype dtype) {
  if (check_sizes(n, E, V, dtype) != LVX_OK || !entries_ok(K)) return 0;
  const EntryPlan e = entries_of(n, V, K);
  const size_t fwd = e.fwd + align_up(plan_of(n, E, V, dtype).fwd), bwd = e.bwd + lvx_xent_workspace_bytes(n, E, V, dtype);
  return fwd > bwd ? fwd : bwd;
}

lvx_status lvx_distil_fwd(const lvx_distil* p, lvx_dtype dtype, const void* x, const void* w, const int64_t* ids, const void* teacher,
                          lvx_dtype teacher_dtype, float* loss, float* lse, float* ln_p, void* workspace, size_t workspace_bytes, void* hip_stream) {
  lvx_status st = distil_check(p, dtype, ids, teacher, teacher_dtype, loss, lse, ln_p, workspace);
  if (st != LVX_OK) return st;
  const size_t own = entries_of(p->n, p->V, p->K).fwd;
  const lvx_xent product = {p->n, p->V, p->E, p->x_ss};
  XentArgs a;
  Plan plan;
  st = xent_args(&product, dtype, x, w, (const int64_t*)workspace, (char*)workspace + own, &a, &plan);
  if (st != LVX_OK) return st;
  if (workspace_bytes < own || workspace_bytes - own < plan.fwd) return LVX_ERR_WORKSPACE;
  distil_args(p, ids, teacher, teacher_dtype, ln_p, workspace, &a);
  a.loss = loss; a.lse_out = lse;
  return launch_distil_fwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

lvx_status lvx_distil_bwd(const lvx_distil* p, lvx_dtype dtype, const void* x, const void* w, const int64_t* ids, const void* teacher,
                          lvx_dtype teacher_dtype, const float* lse, const float* ln_p, const float* d_loss, void* dx, void* dw, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  lvx_status st = distil_check(p, dtype, ids, teacher, teacher_dtype, d_loss, lse, ln_p, workspace);
  if (st != LVX_OK) return st;
  const size_t own = entries_of(p->n, p->V, p->K).bwd;
  if (workspace_bytes < own) return LVX_ERR_WORKSPACE;
  const lvx_xent product = {p->n, p->V, p->E, p->x_ss};
  XentArgs a;
  st = xent_bwd_args(&product, dtype, x, w, (const int64_t*)workspace, lse, d_loss, dx, dw, (char*)workspace + own, workspace_bytes - own, &a);
  if (st != LVX_OK) return st;
  distil_args(p, ids, teacher, teacher_dtype, (float*)ln_p, workspace, &a);      // (read only)
  return launch_distil_bwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

}  // extern "C"
