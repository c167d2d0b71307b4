// Arguments and host-side launchers of the linear-layer kernels and the activation checkpoints
// (internal to libsmat).
//
// Every product is out[i][j] = sum_r P(i, r) Q(j, r) with an epilogue on out.  An operand is `direct`
// where r runs along its rows, P(i, r) = P[i ld + r], and `transposed` where its rows are r,
// P(i, r) = P[r ld + i]:
//   layer            P = x [m, k] direct        Q = W [n, k] direct        i = m, j = n, r = k
//   data gradient    P = dy [m, k] direct       Q = W [k, n] transposed    i = m, j = n, r = k
//   weight gradient  P = dy [m, n] transposed   Q = x [m, k] transposed    i = n, j = k, r = m
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

enum LinEpilogue : int { kEpiStore = 0, kEpiLayer = 1, kEpiDgrad = 2 };

struct LinProduct {
  const void* p;
  const void* q;
  int64_t ldp, ldq;
  int64_t r;
};

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
  float* partial;
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
};
// Element types by smat_dtype code: 0 = fp32, 1 = bf16.
LinPlan linear_plan(const LinArgs& a, int dtype, LinEpilogue epi);
hipError_t launch_linear(const LinArgs& a, int dtype, LinEpilogue epi, const LinPlan& plan, void* workspace,
                         hipStream_t stream);

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
