// C ABI of the linear-layer products and the activation checkpoints: argument checks and launches.
// Kernels live in smat_linear.hip and smat_ckpt.hip.
#include <algorithm>

#include "smat.h"
#include "smat_check.h"
#include "smat_error.h"
#include "smat_linear.h"

using namespace smat;

namespace {

// Arguments of one call, checked, as the launch takes them.
struct Call {
  smat::LinArgs a{};
  smat::LinPlan plan{};
  bool empty = false;
};

smat_status linear_call(const smat_linear_args* g, Call* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_types(g->dtype, g->act, where)) return st;
  const int64_t dims[] = {g->m, g->n, g->k};
  if (smat_status st = check_dims(dims, 3, where)) return st;
  if ((g->z_codes == nullptr) != (g->z_exps == nullptr) && g->m > 0 && g->n > 0)
    return fail(SMAT_ERR_INVALID, "%s: a checkpoint needs codes and exps", where);
  Array arrays[9];
  int n = 0;
  arrays[n++] = matrix("out", g->out, g->m, g->n, g->ldout, g->dtype, true, true);
  if (g->z_codes) {
    arrays[n++] = codes("z_codes", g->z_codes, g->m, g->n, true);
    arrays[n++] = exps("z_exps", g->z_exps, g->m, g->n, true);
  }
  arrays[n++] = matrix("x", g->x, g->m, g->k, g->ldx, g->dtype);
  arrays[n++] = matrix("w", g->w, g->n, g->k, g->ldw, g->dtype);
  if (g->bias) arrays[n++] = matrix("bias", g->bias, 1, g->n, g->n, g->dtype);
  if (g->mul) arrays[n++] = matrix("mul", g->mul, g->m, g->n, g->ldmul, g->dtype, false, true);
  if (g->residual) arrays[n++] = matrix("residual", g->residual, g->m, g->n, g->ldres, g->dtype, false, true);
  c->empty = g->m == 0 || g->n == 0;
  if (c->empty) return SMAT_OK;
  if (smat_status st = check_arrays(arrays, n, where)) return st;
  if (smat_status st = check_grid(g->m, g->n, where)) return st;
  smat::LinArgs& a = c->a;
  a.prod[0] = smat::LinProduct{g->x, g->w, g->ldx, g->ldw, g->k};
  a.i = g->m;
  a.j = g->n;
  a.out = g->out;
  a.ldout = g->ldout;
  a.bias = g->bias;
  a.mul = g->mul;
  a.ldmul = g->ldmul;
  a.residual = g->residual;
  a.ldres = g->ldres;
  a.codes = g->z_codes;
  a.exps = g->z_exps;
  a.act = g->act;
  c->plan = smat::linear_plan(a, g->dtype, smat::kEpiLayer);
  return SMAT_OK;
}

smat_status dgrad_call(const smat_linear_dgrad_args* g, Call* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_types(g->dtype, g->act, where)) return st;
  const int64_t dims[] = {g->m, g->n, g->k, g->k2};
  if (smat_status st = check_dims(dims, 4, where)) return st;
  c->empty = g->m == 0 || g->n == 0;
  if (c->empty) return SMAT_OK;
  if ((g->z_codes == nullptr) != (g->z_exps == nullptr) || (g->up_codes == nullptr) != (g->up_exps == nullptr))
    return fail(SMAT_ERR_INVALID, "%s: a checkpoint needs codes and exps", where);
  if (!g->z_codes && (g->act != SMAT_ACT_NONE || g->up_codes))
    return fail(SMAT_ERR_INVALID, "%s: an activation or an up checkpoint needs the z checkpoint", where);
  if ((g->up_codes == nullptr) != (g->out_up == nullptr))
    return fail(SMAT_ERR_INVALID, "%s: out_up goes with the up checkpoint", where);
  Array arrays[10];
  int n = 0;
  arrays[n++] = matrix("out", g->out, g->m, g->n, g->ldout, g->dtype, true);
  if (g->out_up) arrays[n++] = matrix("out_up", g->out_up, g->m, g->n, g->ldup, g->dtype, true);
  arrays[n++] = matrix("dy", g->dy, g->m, g->k, g->lddy, g->dtype);
  arrays[n++] = matrix("w", g->w, g->k, g->n, g->ldw, g->dtype);
  arrays[n++] = matrix("dy2", g->dy2, g->m, g->k2, g->lddy2, g->dtype);
  arrays[n++] = matrix("w2", g->w2, g->k2, g->n, g->ldw2, g->dtype);
  if (g->z_codes) {
    arrays[n++] = codes("z_codes", g->z_codes, g->m, g->n);
    arrays[n++] = exps("z_exps", g->z_exps, g->m, g->n);
  }
  if (g->up_codes) {
    arrays[n++] = codes("up_codes", g->up_codes, g->m, g->n);
    arrays[n++] = exps("up_exps", g->up_exps, g->m, g->n);
  }
  if (smat_status st = check_arrays(arrays, n, where)) return st;
  if (smat_status st = check_grid(g->m, g->n, where)) return st;
  smat::LinArgs& a = c->a;
  a.prod[0] = smat::LinProduct{g->dy, g->w, g->lddy, g->ldw, g->k};
  a.prod[1] = smat::LinProduct{g->dy2, g->w2, g->lddy2, g->ldw2, g->k2};
  a.i = g->m;
  a.j = g->n;
  a.out = g->out;
  a.ldout = g->ldout;
  a.z_codes = g->z_codes;
  a.z_exps = g->z_exps;
  a.up_codes = g->up_codes;
  a.up_exps = g->up_exps;
  a.out_up = g->out_up;
  a.ldup = g->ldup;
  a.act = g->act;
  c->plan = smat::linear_plan(a, g->dtype, smat::kEpiDgrad);
  return SMAT_OK;
}

// The workspace of a weight gradient: the product's, and x read back from its checkpoint.
struct WgradCall : Call {
  size_t product = 0, x = 0;
  size_t bytes() const { return product + x; }
};

smat_status wgrad_call(const smat_linear_wgrad_args* g, WgradCall* c, const char* where) {
  if (!g) return fail(SMAT_ERR_INVALID, "%s: args is NULL", where);
  if (smat_status st = check_types(g->dtype, SMAT_ACT_NONE, where)) return st;
  if (g->reserved != 0) return fail(SMAT_ERR_INVALID, "%s: reserved must be 0", where);
  const int64_t dims[] = {g->m, g->n, g->k};
  if (smat_status st = check_dims(dims, 3, where)) return st;
  const bool ckpt = g->x_codes || g->x_exps;
  if (ckpt && (g->x || !g->x_codes || !g->x_exps))
    return fail(SMAT_ERR_INVALID, "%s: x is a matrix or a checkpoint (codes and exps)", where);
  Array arrays[6];
  int n = 0;
  arrays[n++] = matrix("dw", g->dw, g->n, g->k, g->lddw, g->dtype, true);
  if (g->db) arrays[n++] = matrix("db", g->db, 1, g->n, g->n, g->dtype, true);
  arrays[n++] = matrix("dy", g->dy, g->m, g->n, g->lddy, g->dtype);
  if (ckpt) {
    arrays[n++] = codes("x_codes", g->x_codes, g->m, g->k);
    arrays[n++] = exps("x_exps", g->x_exps, g->m, g->k);
  } else {
    arrays[n++] = matrix("x", g->x, g->m, g->k, g->ldx, g->dtype);
  }
  if (smat_status st = check_arrays(arrays, n, where)) return st;
  if (smat_status st = check_grid(g->n, g->k, where)) return st;
  if (smat_status st = check_grid(g->m, g->k, where)) return st;
  smat::LinArgs& a = c->a;
  a.prod[0] = smat::LinProduct{g->dy, g->x, g->lddy, g->ldx, g->m};
  a.i = g->n;
  a.j = g->k;
  a.out = g->dw;
  a.ldout = g->lddw;
  c->empty = g->n == 0 || g->k == 0;
  if (!c->empty) {
    if (ckpt) a.prod[0].ldq = smat::ckpt_blocks(g->k) * smat::kCkptBlock;  // as it is read back into the workspace
    c->plan = smat::linear_plan(a, g->dtype, smat::kEpiStore);
    c->product = round16(c->plan.workspace);
    if (ckpt) c->x = (size_t)g->m * (size_t)(smat::ckpt_blocks(g->k) * smat::kCkptBlock) * dtype_bytes(g->dtype);
  }
  return SMAT_OK;
}

}  // namespace

// ------------------------------------------------------------------ checkpoints
extern "C" smat_status smat_ckpt_write(const void* x, int64_t ldx, smat_dtype dtype, int64_t rows, int64_t cols,
                                       int8_t* z_codes, uint8_t* z_exps, hipStream_t stream) {
  const char* where = "smat_ckpt_write";
  if (smat_status st = check_types(dtype, SMAT_ACT_NONE, where)) return st;
  const int64_t dims[] = {rows, cols};
  if (smat_status st = check_dims(dims, 2, where)) return st;
  if (rows == 0 || cols == 0) return SMAT_OK;
  const Array arrays[] = {codes("codes", z_codes, rows, cols, true), exps("exps", z_exps, rows, cols, true),
                          matrix("x", x, rows, cols, ldx, dtype)};
  if (smat_status st = check_arrays(arrays, 3, where)) return st;
  if (smat_status st = check_grid(rows, cols, where)) return st;
  SMAT_HIP(smat::launch_ckpt_write(x, ldx, rows, cols, dtype, z_codes, z_exps, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_ckpt_read(const int8_t* z_codes, const uint8_t* z_exps, const int8_t* up_codes,
                                      const uint8_t* up_exps, smat_act act, smat_dtype dtype, int64_t rows,
                                      int64_t cols, void* out, int64_t ldout, hipStream_t stream) {
  const char* where = "smat_ckpt_read";
  if (smat_status st = check_types(dtype, act, where)) return st;
  const int64_t dims[] = {rows, cols};
  if (smat_status st = check_dims(dims, 2, where)) return st;
  if (rows == 0 || cols == 0) return SMAT_OK;
  if ((up_codes == nullptr) != (up_exps == nullptr))
    return fail(SMAT_ERR_INVALID, "%s: a checkpoint needs codes and exps", where);
  Array arrays[5] = {matrix("out", out, rows, cols, ldout, dtype, true), codes("codes", z_codes, rows, cols),
                     exps("exps", z_exps, rows, cols)};
  int n = 3;
  if (up_codes) {
    arrays[n++] = codes("up_codes", up_codes, rows, cols);
    arrays[n++] = exps("up_exps", up_exps, rows, cols);
  }
  if (smat_status st = check_arrays(arrays, n, where)) return st;
  if (smat_status st = check_grid(rows, cols, where)) return st;
  SMAT_HIP(smat::launch_ckpt_read(z_codes, z_exps, up_codes, up_exps, act, rows, cols, dtype, out, ldout, stream));
  return SMAT_OK;
}

// ------------------------------------------------------------------ products
extern "C" smat_status smat_linear_workspace_bytes(const smat_linear_args* args, size_t* bytes) {
  Call c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_linear_workspace_bytes: bytes is NULL");
  if (smat_status st = linear_call(args, &c, "smat_linear_workspace_bytes")) return st;
  *bytes = c.plan.workspace;
  return SMAT_OK;
}

extern "C" smat_status smat_linear(const smat_linear_args* args, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  Call c;
  if (smat_status st = linear_call(args, &c, "smat_linear")) return st;
  if (c.empty) return SMAT_OK;
  if (smat_status st = check_workspace(workspace, workspace_bytes, c.plan.workspace, "smat_linear")) return st;
  SMAT_HIP(smat::launch_linear(c.a, args->dtype, smat::kEpiLayer, c.plan, workspace, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_linear_dgrad_workspace_bytes(const smat_linear_dgrad_args* args, size_t* bytes) {
  Call c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_linear_dgrad_workspace_bytes: bytes is NULL");
  if (smat_status st = dgrad_call(args, &c, "smat_linear_dgrad_workspace_bytes")) return st;
  *bytes = c.plan.workspace;
  return SMAT_OK;
}

extern "C" smat_status smat_linear_dgrad(const smat_linear_dgrad_args* args, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
  Call c;
  if (smat_status st = dgrad_call(args, &c, "smat_linear_dgrad")) return st;
  if (c.empty) return SMAT_OK;
  if (smat_status st = check_workspace(workspace, workspace_bytes, c.plan.workspace, "smat_linear_dgrad")) return st;
  SMAT_HIP(smat::launch_linear(c.a, args->dtype, smat::kEpiDgrad, c.plan, workspace, stream));
  return SMAT_OK;
}

extern "C" smat_status smat_linear_wgrad_workspace_bytes(const smat_linear_wgrad_args* args, size_t* bytes) {
  WgradCall c;
  if (!bytes) return fail(SMAT_ERR_INVALID, "smat_linear_wgrad_workspace_bytes: bytes is NULL");
  if (smat_status st = wgrad_call(args, &c, "smat_linear_wgrad_workspace_bytes")) return st;
  *bytes = c.bytes();
  return SMAT_OK;
}

extern "C" smat_status smat_linear_wgrad(const smat_linear_wgrad_args* args, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
  WgradCall c;
  if (smat_status st = wgrad_call(args, &c, "smat_linear_wgrad")) return st;
  if (smat_status st = check_workspace(workspace, workspace_bytes, c.bytes(), "smat_linear_wgrad")) return st;
  char* ws = static_cast<char*>(workspace);
  if (args->db && args->n > 0)
    SMAT_HIP(smat::launch_column_sum(args->dy, args->lddy, args->m, args->n, args->dtype, args->db, stream));
  if (c.empty) return SMAT_OK;
  if (c.x) {
    void* x = ws + c.product;
    SMAT_HIP(smat::launch_ckpt_read(args->x_codes, args->x_exps, nullptr, nullptr, SMAT_ACT_NONE, args->m, args->k,
                                    args->dtype, x, c.a.prod[0].ldq, stream));
    c.a.prod[0].q = x;
  }
  SMAT_HIP(smat::launch_linear(c.a, args->dtype, smat::kEpiStore, c.plan, workspace, stream));
  return SMAT_OK;
}
