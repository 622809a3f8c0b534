// C ABI of the norms and of the packed form (see include/lvx.h): argument validation on the host and launches on the
// caller's stream.
#include "../../include/lvx.h"
#include "lvx_internal.h"
#include "lvx_packed.h"

using namespace lvx;

namespace {

constexpr size_t ALIGN = 256;

// an element of the type lies at p, and at every row
bool aligned_for(const void* p, lvx_dtype dtype) { return (uintptr_t)p % (dtype == LVX_F32 ? 4 : 2) == 0; }

lvx_status check_rows(int64_t n, int32_t E, int64_t stride, lvx_dtype dtype) {
  if (dtype != LVX_F32 && dtype != LVX_BF16) return LVX_ERR_DTYPE;
  if (n < 1 || E < 1 || n > INT32_MAX || E > (1 << 24)) return LVX_ERR_SHAPE;
  return stride < E ? LVX_ERR_STRIDE : LVX_OK;
}

lvx_status pack_args(int64_t n, int32_t E, int64_t x_ss, lvx_dtype dtype, const void* x, const lvx_packed* p, NormArgs* a) {
  if (!x || !p || !p->q || !p->e) return LVX_ERR_NULL;
  const lvx_status st = check_rows(n, E, x_ss, dtype);
  if (st != LVX_OK) return st;
  if (!aligned_for(x, dtype)) return LVX_ERR_STRIDE;
  *a = NormArgs{};
  a->n = n; a->E = E; a->x_ss = a->y_ss = x_ss;
  a->q = p->q; a->b = p->e;
  a->n_cu = device_cu_count();
  return LVX_OK;
}

lvx_status norm_args(const lvx_norm* p, lvx_dtype dtype, NormArgs* a) {
  if (!p) return LVX_ERR_NULL;
  lvx_status st = check_rows(p->n, p->E, p->x_ss, dtype);
  if (st == LVX_OK) st = check_rows(p->n, p->E, p->y_ss, dtype);
  if (st != LVX_OK) return st;
  if (!(p->eps > 0.f)) return LVX_ERR_SHAPE;
  *a = NormArgs{};
  a->n = p->n; a->E = p->E; a->rms = p->rms != 0; a->x_ss = p->x_ss; a->y_ss = p->y_ss; a->eps = p->eps;
  a->n_cu = device_cu_count();
  return LVX_OK;
}

}  // namespace

extern "C" {

lvx_status lvx_pack(int64_t n, int32_t E, int64_t x_ss, lvx_dtype dtype, const void* x, const lvx_packed* to, void* hip_stream) {
  NormArgs a;
  const lvx_status st = pack_args(n, E, x_ss, dtype, x, to, &a);
  if (st != LVX_OK) return st;
  a.x = x;
  return launch_pack(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

lvx_status lvx_unpack(int64_t n, int32_t E, int64_t x_ss, lvx_dtype dtype, const lvx_packed* from, void* x, void* hip_stream) {
  NormArgs a;
  const lvx_status st = pack_args(n, E, x_ss, dtype, x, from, &a);
  if (st != LVX_OK) return st;
  a.y = x;
  return launch_unpack(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

lvx_status lvx_norm_fwd(const lvx_norm* p, lvx_dtype dtype, const void* x, const lvx_packed* packed, const void* gamma,
                        const void* beta, void* y, float* stats, void* hip_stream) {
  NormArgs a;
  const lvx_status st = norm_args(p, dtype, &a);
  if (st != LVX_OK) return st;
  if ((!x && !packed) || (packed && (!packed->q || !packed->e)) || !gamma || !y || !stats) return LVX_ERR_NULL;
  if (!aligned_for(x, dtype) || !aligned_for(y, dtype) || !aligned_for(gamma, dtype) || !aligned_for(beta, dtype) ||
      (uintptr_t)stats % 4 != 0)
    return LVX_ERR_STRIDE;
  if (x == y && p->x_ss != p->y_ss && p->n > 1) return LVX_ERR_STRIDE;
  a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.stats = stats;
  if (packed) { a.q = packed->q; a.b = packed->e; }
  return launch_norm_fwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

size_t lvx_norm_workspace_bytes(int64_t n, int32_t E) {
  if (n < 1 || E < 1 || n > INT32_MAX || E > (1 << 24)) return 0;
  return ((size_t)norm_parts(n, E) * 2 * E * sizeof(float) + ALIGN - 1) / ALIGN * ALIGN;
}

lvx_status lvx_norm_bwd(const lvx_norm* p, lvx_dtype dtype, const void* x, const lvx_packed* packed, const void* gamma,
                        const float* stats, const void* dy, void* dx, float* dgamma, float* dbeta, void* workspace,
                        size_t workspace_bytes, void* hip_stream) {
  NormArgs a;
  const lvx_status st = norm_args(p, dtype, &a);
  if (st != LVX_OK) return st;
  if ((!x && !packed) || (packed && (!packed->q || !packed->e)) || !gamma || !stats || !dy || (!dx && !dgamma && !dbeta))
    return LVX_ERR_NULL;
  if (x && packed) return LVX_ERR_SHAPE;             // (which of the two was normalised?)
  if (!aligned_for(x, dtype) || !aligned_for(dy, dtype) || !aligned_for(dx, dtype) || !aligned_for(gamma, dtype) ||
      (uintptr_t)stats % 4 != 0 || (uintptr_t)dgamma % 4 != 0 || (uintptr_t)dbeta % 4 != 0)
    return LVX_ERR_STRIDE;
  if (dx == dy && p->x_ss != p->y_ss && p->n > 1) return LVX_ERR_STRIDE;
  a.x = x; a.gamma = gamma; a.stats_in = stats; a.dy = dy; a.dx = dx; a.dgamma = dgamma; a.dbeta = dbeta;
  if (packed) { a.q = packed->q; a.b = packed->e; }
  if (dgamma || dbeta) {
    if (!workspace || (uintptr_t)workspace % ALIGN != 0 || workspace_bytes < lvx_norm_workspace_bytes(p->n, p->E)) return LVX_ERR_WORKSPACE;
    a.part = (float*)workspace;
    a.parts = norm_parts(p->n, p->E);
  }
  return launch_norm_bwd(a, dtype == LVX_F32, (hipStream_t)hip_stream) == hipSuccess ? LVX_OK : LVX_ERR_HIP;
}

}  // extern "C"
