// Arguments and host-side launchers of what a decoder has beside its linear layers: norms, the token embedding, and
// the output layer with its loss (internal to libsmat).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "smat_linear.h"

namespace smat {

// ---------------------------------------------------------------- norms
struct NormArgs {
  const void* x;
  int64_t ldx;
  const void* w;  // NULL: ones
  const void* b;  // NULL: zeros
  void* y;
  int64_t ldy;
  float* mean;
  float* rstd;
  int64_t m, n;
  float eps;
  int32_t layer, wdtype;
};
hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t stream);

struct NormGradArgs {
  const void* dy;
  int64_t lddy;
  const void* x;
  int64_t ldx;
  const void* w;
  const float* mean;
  const float* rstd;
  void* dx;  // NULL: not wanted, as dw and db
  int64_t lddx;
  void* dw;
  void* db;
  float* partial;  // [1 or 2][blocks][n]
  int64_t m, n;
  int32_t layer, wdtype, blocks;
};
// Blocks that share the rows, each with its sums of dw and db, and the bytes of `partial` for so many outputs.
int32_t norm_grad_blocks(int64_t m, int64_t n);
size_t norm_grad_partial(int64_t m, int64_t n, int outputs);
hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t stream);

// ---------------------------------------------------------------- embedding
struct EmbedArgs {
  const void* table;
  int64_t ldt, rows;
  const int64_t* ids;
  void* out;
  int64_t ldout, m, d;
  float scale;
};
hipError_t launch_embed(const EmbedArgs& a, int table_dtype, int dtype, hipStream_t stream);

struct EmbedGradArgs {
  const void* dy;
  int64_t lddy;
  const int64_t* ids;
  void* dtable;
  int64_t ldt, rows, m, d;
  int64_t padding;
  float scale;
  int32_t accumulate;
};
// Where the sorted tokens and the sums of cut runs lie in the workspace.
struct EmbedGradPlan {
  int64_t chunk, chunks;  // sorted tokens that one wave sums, and how many such there are
  int32_t bits, passes;   // of the ids, and of the sort
  int64_t tiles;          // of the sort, or 1
  size_t keys[2], places[2], counts, partial, workspace;
};
EmbedGradPlan embed_grad_plan(const EmbedGradArgs& a);
hipError_t launch_embed_grad(const EmbedGradArgs& a, int dtype, int table_dtype, const EmbedGradPlan& plan,
                             void* workspace, hipStream_t stream);

// ---------------------------------------------------------------- output layer with its loss
struct XentArgs {
  const void* x;
  const void* w;
  int64_t ldx, ldw, m, n, k;
  const int64_t* targets;
  int64_t ignore;
  float* loss;
  float* lse;
  float* lse_low;  // or NULL
  float* totals;  // sum of the losses, rows that count, their mean; or NULL
};
struct XentPlan {
  LinPlan logits;
  size_t stats, target_z, workspace;
};
XentPlan xent_plan(const XentArgs& a, int dtype);
hipError_t launch_xent(const XentArgs& a, int dtype, const XentPlan& plan, void* workspace, hipStream_t stream);

struct XentGradArgs {
  const void* x;
  const void* w;
  int64_t ldx, ldw, m, n, k;
  const int64_t* targets;
  int64_t ignore;
  const float* lse;
  const float* lse_low;  // or NULL
  const float* row_scale;
  const float* scale;
  const float* totals;
  void* dx;  // NULL: not wanted, as dw
  int64_t lddx;
  void* dw;
  int64_t lddw;
};
// Pieces of `width` columns of the vocabulary, the last one narrower: how each piece's products are computed.
struct XentGradPlan {
  int64_t width, pieces;
  int32_t pack;  // each piece of W is copied to 16-byte rows for its products; x always is
  int32_t low;   // what rounding dz to bf16 leaves is kept too, behind dz, and multiplied
  int32_t some;  // the products take the rows with a target only, in order; x is copied so
  int64_t first;  // with `some`: the logits' first part has so many rows, which stay its own; 0: any row may be in either part
  LinPlan logits[2], dx[2], dw[2];  // of a whole piece and of the last one
  size_t dz, sum, x, w, rows, workspace;  // behind the products' own
};
XentGradPlan xent_grad_plan(const XentGradArgs& a, int dtype);
hipError_t launch_xent_grad(const XentGradArgs& a, int dtype, const XentGradPlan& plan, void* workspace, hipStream_t stream);

}  // namespace smat
