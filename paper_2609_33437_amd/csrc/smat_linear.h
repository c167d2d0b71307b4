// Arguments and host-side launchers of the linear-layer kernels and the activation checkpoints
// (internal to libsmat).
//
// Every product is out[i][j] = sum_r P(i, r) Q(j, r) with an epilogue on out.  An operand is `direct`
// where r runs along its rows, P(i, r) = P[i ld + r], and `transposed` where its rows are r,
// P(i, r) = P[r ld + i]:
//   layer            P = x [m, k] direct        Q = W [n, k] direct        i = m, j = n, r = k
//   data gradient    P = dy [m, k] direct       Q = W [k, n] transposed    i = m, j = n, r = k
//   weight gradient  P = dy [m, n] transposed   Q = x [m, k] transposed    i = n, j = k, r = m
// The output layer's loss takes the layer's form for its logits, whose rows its epilogues reduce (kEpiXent) or turn into
// gradients (kEpiXentGrad), and the other two for dx (kEpiSum) and dW (kEpiScaled) of pieces of the vocabulary.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace smat {

constexpr int kCkptBlock = 32;  // elements along a row that share a checkpoint's power of two
inline int64_t ckpt_blocks(int64_t cols) { return (cols + kCkptBlock - 1) / kCkptBlock; }

// A launch whose grid has 2^32 threads or more in a dimension does less than it was asked, without an error.
constexpr int64_t kMaxThreads = INT64_C(0xFFFFFFFF);
// Grids of kernels that may need more: rows of 2^20 blocks, numbered by wide_block() in the kernel.
constexpr int kWideShift = 20;
inline dim3 wide_grid(int64_t blocks) {
  constexpr int64_t kRow = (int64_t)1 << kWideShift;
  return blocks <= kRow ? dim3((uint32_t)blocks) : dim3((uint32_t)kRow, (uint32_t)((blocks + kRow - 1) >> kWideShift));
}

enum LinEpilogue : int { kEpiStore = 0, kEpiLayer = 1, kEpiDgrad = 2, kEpiXent = 3, kEpiXentGrad = 4, kEpiSum = 5, kEpiScaled = 6 };
constexpr bool p_transposed(int epi) { return epi == kEpiStore || epi == kEpiScaled; }
constexpr bool q_transposed(int epi) { return !(epi == kEpiLayer || epi == kEpiXent || epi == kEpiXentGrad); }

struct LinProduct {
  const void* p;
  const void* q;
  int64_t ldp, ldq;
  int64_t r;
};

// What the linear layers' products read comes first, as close as it was without the loss's fields: with them before `splits` and
// a wider LinProduct 1001 x 2001 x 2001 by way of registers took 31.2 us (30.6), fp32 1223 x 1378 x 1001 56.7 us (56.1).
struct LinArgs {
  LinProduct prod[2];  // the products that are summed; prod[1].r == 0 where there is one
  int64_t i, j;
  void* out;
  int64_t ldout;
  // layer: out = act(v + bias) (.) mul + residual, codes and exps of v + bias
  const void* bias;
  const void* mul;
  const void* residual;
  int64_t ldmul, ldres;
  int8_t* codes;
  uint8_t* exps;
  // data gradient: act'(z^) from z, u^ from up; out_up = v (.) act(z^)
  const int8_t* z_codes;
  const uint8_t* z_exps;
  const int8_t* up_codes;
  const uint8_t* up_exps;
  void* out_up;
  int64_t ldup;
  int32_t act;
  // sums of `splits` ranges of r, joined by a second kernel: [splits][i][j rounded up to 8] fp32
  int32_t splits;
  int32_t p_clean;  // P's rows hold finite values, whatever they are, from their end to the next 16 bytes
  float* partial;
  // cross entropy of logits v, columns col0 .. col0 + j of `classes` ones: the largest value and the sum of exponentials of
  // each tile's columns of a row, and the target's logit; or out = (exp(v - lse - lse_low) - [column is the target]) row_scale
  const int64_t* targets;
  int64_t ignore, classes, col0;
  float* stats;  // [i][stat_ld][2]
  int64_t stat_ld;
  float* target_z;
  const float* lse;
  const float* lse_low;    // NULL: 0
  const float* row_scale;  // NULL: 1
  void* out_low;  // what rounding out to bf16 left, in bf16; or NULL
  // out = s (v + sum_in), zeros in rows without a target (targets not NULL), or sum_out = v + sum_in (NULL: 0), with s = scale[0] / totals[1] (NULL: 1)
  const float* sum_in;
  float* sum_out;
  int64_t ldsum;
  const float* scale;
  const float* totals;
  // rows that there are of the i (of the r of kEpiScaled) that were planned, in device memory, or NULL: all; row_from: the part's
  // first; out_rows: where kEpiSum writes them, or NULL: as they are numbered
  const int32_t* count;
  const int32_t* out_rows;
  int64_t row_from;
  // of kEpiXentGrad in two parts that sum in different orders: how many of `count` are the first part's, or NULL: as many as it
  // has rows.  The second part's follow them.
  const int32_t* first_count;
  // of kEpiSum: rows of a tile and the ranges of r that may be made, for fewer rows than planned; the block's own range
  int32_t tile_rows, most_splits, range;
};

// How a product is computed: rows [0, part[0].rows) of out by one launch (and a join), the rest by another.
struct LinPart {
  int64_t rows;
  int32_t form;    // which tile (smat_linear.hip)
  int32_t splits;  // ranges of r
};
struct LinPlan {
  LinPart part[2];
  int32_t parts;
  int32_t direct;    // operands go to LDS without passing registers
  int32_t pack;      // bits: operands copied to 16-byte rows first (P, Q of prod[0], then of prod[1])
  size_t packed[4];  // where in the workspace
  size_t workspace;  // bytes
  double us;         // estimated
};
// Element types by smat_dtype code: 0 = fp32, 1 = bf16.
// With `like`, a plan of as many rows and as long sums, each row's sums are formed in that plan's order, to the same bits.
LinPlan linear_plan(const LinArgs& a, int dtype, LinEpilogue epi, const LinPlan* like = nullptr);
// Whether a plan's parts sum in the same order.
bool one_order(const LinPlan& plan);
// Columns that one pair of a row's stats covers in a part of a plan.
int64_t stat_columns(const LinPart& part);
hipError_t launch_linear(const LinArgs& a, int dtype, LinEpilogue epi, const LinPlan& plan, void* workspace,
                         hipStream_t stream);

// Copies `rows` runs of `run` elements to rows of packed_stride(run) elements, whole 16 bytes with zeros at their ends.
int64_t packed_stride(int64_t run, int dtype);
hipError_t launch_pack(const void* from, int64_t ld, int64_t rows, int64_t run, int dtype, void* to, hipStream_t stream);
constexpr double pack_us(double bytes) { return 3.0 + 2.0 * bytes / 5.0e6; }

// db[j] = sum_i dy[i][j] for dy [rows, cols].
hipError_t launch_column_sum(const void* dy, int64_t ld, int64_t rows, int64_t cols, int dtype, void* db,
                             hipStream_t stream);

hipError_t launch_ckpt_write(const void* x, int64_t ld, int64_t rows, int64_t cols, int dtype, int8_t* codes,
                             uint8_t* exps, hipStream_t stream);
// out = act(z^), or act(z^) (.) u^ with up_codes.
hipError_t launch_ckpt_read(const int8_t* codes, const uint8_t* exps, const int8_t* up_codes, const uint8_t* up_exps,
                            int act, int64_t rows, int64_t cols, int dtype, void* out, int64_t ldout,
                            hipStream_t stream);

}  // namespace smat
