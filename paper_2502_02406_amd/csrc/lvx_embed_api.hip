// C ABI of the embedding lookup (see include/lvx.h): argument validation on the host, workspace carving, and launches on the caller's
// stream.
#include "../../include/lvx.h"
#include "lvx_internal.h"

using namespace lvx;

namespace {

constexpr size_t ALIGN = 256;
size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
bool aligned(const void* p, size_t by) { return (uintptr_t)p % by == 0; }

bool sizes_ok(int64_t n, int32_t E, int64_t V) { return n >= 1 && E >= 1 && V >= 1 && n <= (1 << 28) && V <= (1 << 28) && E <= (1 << 20); }

// `rows`: y or d_y, `table`: the table or its gradient
lvx_status embed_args(const lvx_embed* p, lvx_dtype dtype, const int64_t* ids, const void* rows, const void* table, EmbedArgs* a) {
  if (!p || !ids || !rows || !table) return LVX_ERR_NULL;
  if (dtype != LVX_F32 && dtype != LVX_BF16) return LVX_ERR_DTYPE;
  if (!sizes_ok(p->n, p->E, p->V)) return LVX_ERR_SHAPE;
  const int64_t el = dtype == LVX_F32 ? 4 : 2;
  if (p->y_ss < p->E || p->y_ss > ((int64_t)1 << 40) / p->n || !aligned(rows, el) || !aligned(table, el) || !aligned(ids, 8)) return LVX_ERR_STRIDE;
  // (what is read in place of what is written, or the other way round)
  if (rows_meet((int64_t)rows, p->n, p->y_ss * el, p->E * el, (int64_t)table, p->V * p->E * el)) return LVX_ERR_STRIDE;
  *a = EmbedArgs{};
  a->ids = ids;
  a->n = p->n; a->V = p->V; a->y_ss = p->y_ss; a->E = p->E; a->scale = p->scale;
  a->n_cu = device_cu_count();
  return LVX_OK;
}

struct Plan { size_t list[4], hist, top, long_list, part, all; };
Plan plan_of(int64_t n, int32_t E) {
  Plan p;
  size_t at = align_up(sizeof(EmbedHead));
  for (size_t& l : p.list) { l = at; at += align_up(n * sizeof(int)); }
  p.hist = at; at += (size_t)EMBED_BLOCKS * EMBED_DIGITS * sizeof(int);
  p.top = at; at += align_up((EMBED_TOPS + 1) * sizeof(int));
  p.long_list = at; at += align_up((EMBED_LISTS + 1) * embed_list_room(n) * sizeof(int2));
  p.part = at; at += align_up(embed_part_room(n, E));
  p.all = at;
  return p;
}

}  // namespace

extern "C" {

lvx_status lvx_embed_fwd(const lvx_embed* p, lvx_dtype dtype, const void* table, const int64_t* ids, void* y, void* hip_stream) {
  EmbedArgs a;
  const lvx_status st = embed_args(p, dtype, ids, y, table, &a);
  if (st != LVX_OK) return st;
  a.table = table; a.y = y;
  return launch_embed_fwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

size_t lvx_embed_workspace_bytes(int64_t n, int32_t E, int64_t V) { return sizes_ok(n, E, V) ? plan_of(n, E).all : 0; }

lvx_status lvx_embed_bwd(const lvx_embed* p, lvx_dtype dtype, const void* d_y, const int64_t* ids, void* d_table, int accumulate,
                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  EmbedArgs a;
  const lvx_status st = embed_args(p, dtype, ids, d_y, d_table, &a);
  if (st != LVX_OK) return st;
  const Plan plan = plan_of(p->n, p->E);
  if (!workspace || !aligned(workspace, ALIGN) || workspace_bytes < plan.all) return LVX_ERR_WORKSPACE;
  const auto at = [&](size_t o) -> char* { return (char*)workspace + o; };
  a.d_y = d_y; a.d_table = d_table; a.accumulate = accumulate != 0;
  a.head = (EmbedHead*)workspace;
  for (int i = 0; i < 2; ++i) {
    a.key[i] = (int*)at(plan.list[i]);
    a.tok[i] = (int*)at(plan.list[2 + i]);
  }
  a.hist = (int*)at(plan.hist); a.top = (int*)at(plan.top); a.long_list = (int2*)at(plan.long_list); a.part = (float*)at(plan.part);
  return launch_embed_bwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

}  // extern "C"
