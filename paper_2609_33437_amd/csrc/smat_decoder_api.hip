// C ABI of the norms, the token embedding and the output layer with its loss: argument checks and launches.
// Kernels live in smat_norm.hip, smat_embed.hip and smat_xent.hip.
#include <math.h>

#include "smat.h"
#include "smat_check.h"
#include "smat_decoder.h"
#include "smat_error.h"

using namespace smat;

namespace {

// A call's arrays, as the checks see them.
struct Arrays {
  Array a[12];
  int n = 0;
  void add(const Array& x) { a[n++] = x; }
  void vector(const char* what, const void* p, int64_t count, int64_t bytes, bool out = false) {
    add(Array{what, p, 1, count * bytes, count * bytes, (size_t)bytes, out, false});
  }
  // The workspace too, apart from everything else.
  smat_status check(const char* where) const { return check_arrays(a, n, where); }
  smat_status check_with(void* workspace, size_t have, size_t need, const char* where) {
    if (smat_status st = check_workspace(workspace, have, need, where)) return st;
    if (need) add(Array{"workspace", workspace, 1, (int64_t)need, (int64_t)need, 16, true, false});
    return check(where);
  }
};

smat_status check_dtype(int dtype, const char* where) { return check_types(dtype, SMAT_ACT_NONE, where); }

// ---------------------------------------------------------------- norms
smat_status norm_call(const smat_norm_args* g, NormArgs* a, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_dtype(g->dtype, where)) return st;
  if (smat_status st = check_dtype(g->wdtype, where)) return st;
  if (g->kind != SMAT_NORM_LAYER && g->kind != SMAT_NORM_RMS) return fail(SMAT_ERR_INVALID, "%s: unknown kind %d", where, g->kind);
  if (!(g->eps >= 0.f) || !isfinite(g->eps)) return fail(SMAT_ERR_INVALID, "%s: eps must be finite and >= 0", where);
  const int64_t dims[] = {g->m, g->n};
  if (smat_status st = check_dims(dims, 2, where)) return st;
  Arrays arrays;
  arrays.add(matrix("y", g->y, g->m, g->n, g->ldy, g->dtype, true));
  if (g->mean) arrays.vector("mean", g->mean, g->n ? g->m : 0, 4, true);
  if (g->rstd) arrays.vector("rstd", g->rstd, g->n ? g->m : 0, 4, true);
  arrays.add(matrix("x", g->x, g->m, g->n, g->ldx, g->dtype));
  if (g->weight) arrays.vector("weight", g->weight, g->n, (int64_t)dtype_bytes(g->wdtype));
  if (g->bias) arrays.vector("bias", g->bias, g->n, (int64_t)dtype_bytes(g->wdtype));
  if (smat_status st = arrays.check(where)) return st;
  if (smat_status st = check_grid(g->m, g->n, where)) return st;
  *a = NormArgs{g->x, g->ldx, g->weight, g->bias, g->y, g->ldy, g->mean, g->rstd, g->m, g->n, g->eps,
                g->kind == SMAT_NORM_LAYER, g->wdtype};
  return SMAT_OK;
}

struct NormGradCall {
  NormGradArgs a{};
  Arrays arrays;
  size_t workspace = 0;
};

smat_status norm_grad_call(const smat_norm_grad_args* g, NormGradCall* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_dtype(g->dtype, where)) return st;
  if (smat_status st = check_dtype(g->wdtype, where)) return st;
  if (g->reserved != 0) return fail(SMAT_ERR_INVALID, "%s: reserved must be 0", where);
  if (g->kind != SMAT_NORM_LAYER && g->kind != SMAT_NORM_RMS) return fail(SMAT_ERR_INVALID, "%s: unknown kind %d", where, g->kind);
  const int64_t dims[] = {g->m, g->n};
  if (smat_status st = check_dims(dims, 2, where)) return st;
  const int64_t rows = g->n ? g->m : 0, wb = (int64_t)dtype_bytes(g->wdtype);
  Arrays& arrays = c->arrays;
  if (g->dx) arrays.add(matrix("dx", g->dx, g->m, g->n, g->lddx, g->dtype, true));
  if (g->dweight) arrays.vector("dweight", g->dweight, g->n, wb, true);
  if (g->dbias) arrays.vector("dbias", g->dbias, g->n, wb, true);
  arrays.add(matrix("dy", g->dy, g->m, g->n, g->lddy, g->dtype));
  arrays.add(matrix("x", g->x, g->m, g->n, g->ldx, g->dtype));
  if (g->weight) arrays.vector("weight", g->weight, g->n, wb);
  if (g->kind == SMAT_NORM_LAYER) arrays.vector("mean", g->mean, rows, 4);
  arrays.vector("rstd", g->rstd, rows, 4);
  if (smat_status st = arrays.check(where)) return st;
  if (smat_status st = check_grid(g->m, g->n, where)) return st;
  c->a = NormGradArgs{g->dy, g->lddy, g->x, g->ldx, g->weight, g->mean, g->rstd, g->dx, g->lddx, g->dweight, g->dbias,
                      nullptr, g->m, g->n, g->kind == SMAT_NORM_LAYER, g->wdtype, norm_grad_blocks(g->m, g->n)};
  c->workspace = round16(norm_grad_partial(g->m, g->n, (g->dweight ? 1 : 0) + (g->dbias ? 1 : 0)));
  return SMAT_OK;
}

// ---------------------------------------------------------------- embedding
struct EmbedGradCall {
  EmbedGradArgs a{};
  EmbedGradPlan plan{};
  Arrays arrays;
};

smat_status embed_grad_call(const smat_embed_grad_args* g, EmbedGradCall* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_dtype(g->dtype, where)) return st;
  if (smat_status st = check_dtype(g->table_dtype, where)) return st;
  if (!isfinite(g->scale)) return fail(SMAT_ERR_INVALID, "%s: scale must be finite", where);
  if (g->accumulate != 0 && g->accumulate != 1) return fail(SMAT_ERR_INVALID, "%s: accumulate must be 0 or 1", where);
  const int64_t dims[] = {g->m, g->rows, g->d};
  if (smat_status st = check_dims(dims, 3, where)) return st;
  Arrays& arrays = c->arrays;
  arrays.add(matrix("dtable", g->dtable, g->rows, g->d, g->ldtable, g->table_dtype, true));
  arrays.add(matrix("dy", g->dy, g->m, g->d, g->lddy, g->dtype));
  arrays.vector("ids", g->ids, g->d ? g->m : 0, 8);
  if (smat_status st = arrays.check(where)) return st;
  if (smat_status st = check_grid(g->rows, g->d, where)) return st;
  if (smat_status st = check_grid(g->m, g->d, where)) return st;
  c->a = EmbedGradArgs{g->dy, g->lddy, g->ids, g->dtable, g->ldtable, g->rows, g->m, g->d, g->padding, g->scale, g->accumulate};
  c->plan = embed_grad_plan(c->a);
  return SMAT_OK;
}

// ---------------------------------------------------------------- output layer
smat_status xent_dims(int64_t m, int64_t n, int64_t k, const char* where) {
  const int64_t dims[] = {m, n, k};
  if (smat_status st = check_dims(dims, 3, where)) return st;
  if (n == 0) return fail(SMAT_ERR_INVALID, "%s: there are no classes (n is 0)", where);
  if (smat_status st = check_grid(m, n, where)) return st;
  return check_grid(n, k, where);
}

struct XentCall {
  XentArgs a{};
  XentPlan plan{};
  Arrays arrays;
};

smat_status xent_call(const smat_linear_xent_args* g, XentCall* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_dtype(g->dtype, where)) return st;
  if (g->reserved != 0) return fail(SMAT_ERR_INVALID, "%s: reserved must be 0", where);
  if (smat_status st = xent_dims(g->m, g->n, g->k, where)) return st;
  Arrays& arrays = c->arrays;
  arrays.vector("loss", g->loss, g->m, 4, true);
  arrays.vector("lse", g->lse, g->m, 4, true);
  if (g->totals) arrays.vector("totals", g->totals, 3, 4, true);
  if (g->lse_low) arrays.vector("lse_low", g->lse_low, g->m, 4, true);
  arrays.add(matrix("x", g->x, g->m, g->k, g->ldx, g->dtype));
  arrays.add(matrix("w", g->w, g->n, g->k, g->ldw, g->dtype));
  arrays.vector("targets", g->targets, g->m, 8);
  if (smat_status st = arrays.check(where)) return st;
  c->a = XentArgs{g->x, g->w, g->ldx, g->ldw, g->m, g->n, g->k, g->targets, g->ignore_index, g->loss, g->lse, g->lse_low,
                  g->totals};
  c->plan = xent_plan(c->a, g->dtype);
  return SMAT_OK;
}

struct XentGradCall {
  XentGradArgs a{};
  XentGradPlan plan{};
  Arrays arrays;
};

smat_status xent_grad_call(const smat_linear_xent_grad_args* g, XentGradCall* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_dtype(g->dtype, where)) return st;
  if (g->reserved != 0) return fail(SMAT_ERR_INVALID, "%s: reserved must be 0", where);
  if (smat_status st = xent_dims(g->m, g->n, g->k, where)) return st;
  if (smat_status st = check_grid(g->m, g->k, where)) return st;
  Arrays& arrays = c->arrays;
  if (g->dx) arrays.add(matrix("dx", g->dx, g->m, g->k, g->lddx, g->dtype, true));
  if (g->dw) arrays.add(matrix("dw", g->dw, g->n, g->k, g->lddw, g->dtype, true));
  arrays.add(matrix("x", g->x, g->m, g->k, g->ldx, g->dtype));
  arrays.add(matrix("w", g->w, g->n, g->k, g->ldw, g->dtype));
  arrays.vector("targets", g->targets, g->m, 8);
  arrays.vector("lse", g->lse, g->m, 4);
  if (g->lse_low) arrays.vector("lse_low", g->lse_low, g->m, 4);
  if (g->row_scale) arrays.vector("row_scale", g->row_scale, g->m, 4);
  if (g->scale) arrays.vector("scale", g->scale, 1, 4);
  if (g->totals) arrays.vector("totals", g->totals, 3, 4);
  if (smat_status st = arrays.check(where)) return st;
  c->a = XentGradArgs{g->x, g->w, g->ldx, g->ldw, g->m, g->n, g->k, g->targets, g->ignore_index, g->lse, g->lse_low, g->row_scale,
                      g->scale, g->totals, g->dx, g->lddx, g->dw, g->lddw};
  c->plan = xent_grad_plan(c->a, g->dtype);
  return SMAT_OK;
}

}  // namespace

extern "C" smat_status smat_norm(const smat_norm_args* args, hipStream_t stream) {
  NormArgs a{};
  if (smat_status st = norm_call(args, &a, "smat_norm")) return st;
  if (a.m == 0 || a.n == 0) return SMAT_OK;
  SMAT_HIP(launch_norm(a, args->dtype, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_norm_grad_workspace_bytes(const smat_norm_grad_args* args, size_t* bytes) {
  NormGradCall c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_norm_grad_workspace_bytes: bytes is NULL");
  if (smat_status st = norm_grad_call(args, &c, "smat_norm_grad_workspace_bytes")) return st;
  *bytes = c.workspace;
  return SMAT_OK;
}

extern "C" smat_status smat_norm_grad(const smat_norm_grad_args* args, void* workspace, size_t workspace_bytes,
                                      hipStream_t stream) {
  NormGradCall c;
  if (smat_status st = norm_grad_call(args, &c, "smat_norm_grad")) return st;
  if (smat_status st = c.arrays.check_with(workspace, workspace_bytes, c.workspace, "smat_norm_grad")) return st;
  if (c.a.n == 0) return SMAT_OK;
  c.a.partial = static_cast<float*>(workspace);
  SMAT_HIP(launch_norm_grad(c.a, args->dtype, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_embed(const smat_embed_args* g, hipStream_t stream) {
  const char* where = "smat_embed";
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_dtype(g->dtype, where)) return st;
  if (smat_status st = check_dtype(g->table_dtype, where)) return st;
  if (g->reserved != 0) return fail(SMAT_ERR_INVALID, "%s: reserved must be 0", where);
  if (!isfinite(g->scale)) return fail(SMAT_ERR_INVALID, "%s: scale must be finite", where);
  const int64_t dims[] = {g->m, g->rows, g->d};
  if (smat_status st = check_dims(dims, 3, where)) return st;
  Arrays arrays;
  arrays.add(matrix("out", g->out, g->m, g->d, g->ldout, g->dtype, true));
  arrays.add(matrix("table", g->table, g->rows, g->d, g->ldtable, g->table_dtype));
  arrays.vector("ids", g->ids, g->d ? g->m : 0, 8);
  if (smat_status st = arrays.check(where)) return st;
  if (smat_status st = check_grid(g->m, g->d, where)) return st;
  if (g->m == 0 || g->d == 0) return SMAT_OK;
  const EmbedArgs a{g->table, g->ldtable, g->rows, g->ids, g->out, g->ldout, g->m, g->d, g->scale};
  SMAT_HIP(launch_embed(a, g->table_dtype, g->dtype, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_embed_grad_workspace_bytes(const smat_embed_grad_args* args, size_t* bytes) {
  EmbedGradCall c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_embed_grad_workspace_bytes: bytes is NULL");
  if (smat_status st = embed_grad_call(args, &c, "smat_embed_grad_workspace_bytes")) return st;
  *bytes = c.plan.workspace;
  return SMAT_OK;
}

extern "C" smat_status smat_embed_grad(const smat_embed_grad_args* args, void* workspace, size_t workspace_bytes,
                                       hipStream_t stream) {
  EmbedGradCall c;
  if (smat_status st = embed_grad_call(args, &c, "smat_embed_grad")) return st;
  if (smat_status st = c.arrays.check_with(workspace, workspace_bytes, c.plan.workspace, "smat_embed_grad")) return st;
  if (c.a.rows == 0 || c.a.d == 0) return SMAT_OK;
  SMAT_HIP(launch_embed_grad(c.a, args->dtype, args->table_dtype, c.plan, workspace, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_linear_xent_workspace_bytes(const smat_linear_xent_args* args, size_t* bytes) {
  XentCall c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_linear_xent_workspace_bytes: bytes is NULL");
  if (smat_status st = xent_call(args, &c, "smat_linear_xent_workspace_bytes")) return st;
  *bytes = c.plan.workspace;
  return SMAT_OK;
}

extern "C" smat_status smat_linear_xent(const smat_linear_xent_args* args, void* workspace, size_t workspace_bytes,
                                        hipStream_t stream) {
  XentCall c;
  if (smat_status st = xent_call(args, &c, "smat_linear_xent")) return st;
  if (smat_status st = c.arrays.check_with(workspace, workspace_bytes, c.plan.workspace, "smat_linear_xent")) return st;
  SMAT_HIP(launch_xent(c.a, args->dtype, c.plan, workspace, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_linear_xent_grad_workspace_bytes(const smat_linear_xent_grad_args* args, size_t* bytes) {
  XentGradCall c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_linear_xent_grad_workspace_bytes: bytes is NULL");
  if (smat_status st = xent_grad_call(args, &c, "smat_linear_xent_grad_workspace_bytes")) return st;
  *bytes = c.plan.workspace;
  return SMAT_OK;
}

extern "C" smat_status smat_linear_xent_grad(const smat_linear_xent_grad_args* args, void* workspace,
                                             size_t workspace_bytes, hipStream_t stream) {
  XentGradCall c;
  if (smat_status st = xent_grad_call(args, &c, "smat_linear_xent_grad")) return st;
  if (smat_status st = c.arrays.check_with(workspace, workspace_bytes, c.plan.workspace, "smat_linear_xent_grad")) return st;
  SMAT_HIP(launch_xent_grad(c.a, args->dtype, c.plan, workspace, stream));
  return SMAT_OK;
}
