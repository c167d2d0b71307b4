// The output layer with its cross entropy for gfx950: z = x W^T over a vocabulary, without keeping z.
//
//   lse_i = log sum_j exp z_ij,  loss_i = lse_i - z_i,t_i
//   dz_ij = (exp(z_ij - lse_i) - [j = t_i]) g_i,  dx = s dz W,  dW = s dz^T x
//
// The forward product's epilogue leaves the largest value and the sum of exponentials of each tile's columns of a row, which
// k_xent_rows joins.  The gradient goes through the vocabulary in pieces: a piece's logits again, turned into dz (in the
// call's dtype) by their epilogue, then dz W added to dx in fp32 and dz^T x, which is the piece's part of dW.  So beside
// its outputs a call holds one piece, whatever the vocabulary, for a fourth product beside the three that
// cannot be left out.  s is applied to the fp32 sums of both products, so a mean over many rows costs dz no precision.
#include "smat_decoder.h"
#include "smat_linear_dev.h"

namespace smat {
namespace {

constexpr int kRowThreads = 256;

// A row's log sum of exponentials from its parts, and its loss.
__global__ __launch_bounds__(kRowThreads) void k_xent_rows(XentArgs a, const float* stats, const float* target_z, int64_t from,
                                                           int64_t rows, int64_t parts) {
  __shared__ float tops[kRowThreads / 64], sums[kRowThreads / 64];
  if (wide_block() >= rows) return;
  const f32x2* s = reinterpret_cast<const f32x2*>(stats) + wide_block() * parts;
  const int64_t i = from + wide_block();
  float top = -__builtin_inff(), sum = 0.f;
  for (int64_t k = threadIdx.x; k < parts; k += kRowThreads) {
    const f32x2 v = s[k];
    join_stats(top, sum, v[0], v[1]);
  }
#pragma unroll
  for (int bit = 32; bit > 0; bit >>= 1) join_stats(top, sum, __shfl_xor(top, bit), __shfl_xor(sum, bit));
  if ((threadIdx.x & 63) == 0) {
    tops[threadIdx.x >> 6] = top;
    sums[threadIdx.x >> 6] = sum;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int k = 1; k < kRowThreads / 64; ++k) join_stats(top, sum, tops[k], sums[k]);
  const float lse = logf(sum) + top;
  const int64_t t = a.targets[i];
  a.lse[i] = lse;
  a.loss[i] = t == a.ignore ? 0.f : t < 0 || t >= a.n ? __builtin_nanf("") : lse - target_z[i];
}

// Sum of the losses, rows that count and their mean, in one block and a fixed order, in fp64.
__global__ __launch_bounds__(1024) void k_xent_totals(XentArgs a) {
  __shared__ double sums[16];
  __shared__ int64_t counts[16];
  double sum = 0.0;
  int64_t count = 0;
  for (int64_t i = threadIdx.x; i < a.m; i += 1024) {
    const bool on = a.targets[i] != a.ignore;
    sum += on ? (double)a.loss[i] : 0.0;
    count += on;
  }
#pragma unroll
  for (int bit = 32; bit > 0; bit >>= 1) {
    sum += __shfl_xor(sum, bit);
    count += __shfl_xor((long long)count, bit);
  }
  if ((threadIdx.x & 63) == 0) {
    sums[threadIdx.x >> 6] = sum;
    counts[threadIdx.x >> 6] = count;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int k = 1; k < 16; ++k) {
    sum += sums[k];
    count += counts[k];
  }
  a.totals[0] = (float)sum;
  a.totals[1] = (float)count;
  a.totals[2] = (float)(sum / (double)count);  // NaN where no row counts
}

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }

LinArgs logits_args(const XentArgs& a, void* workspace, const XentPlan& plan) {
  LinArgs l{};
  l.prod[0] = LinProduct{a.x, a.w, a.ldx, a.ldw, a.k};
  l.i = a.m;
  l.j = a.n;
  l.targets = a.targets;
  l.ignore = a.ignore;
  l.classes = a.n;
  l.stats = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.stats);
  l.target_z = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.target_z);
  return l;
}
}  // namespace

XentPlan xent_plan(const XentArgs& a, int dtype) {
  XentPlan p{};
  if (a.m == 0) return p;
  p.logits = linear_plan(logits_args(a, nullptr, p), dtype, kEpiXent);
  p.stats = round16(p.logits.workspace);
  size_t pairs = 0;
  for (int k = 0; k < p.logits.parts; ++k)
    pairs += (size_t)p.logits.part[k].rows * (size_t)div_up(a.n, stat_columns(p.logits.part[k]));
  p.target_z = p.stats + round16(pairs * 8);
  p.workspace = p.target_z + round16((size_t)a.m * 4);
  return p;
}

hipError_t launch_xent(const XentArgs& a, int dtype, const XentPlan& plan, void* workspace, hipStream_t stream) {
  hipError_t e = hipSuccess;
  if (a.m > 0) {
    const LinArgs l = logits_args(a, workspace, plan);
    e = launch_linear(l, dtype, kEpiXent, plan.logits, workspace, stream);
    if (e != hipSuccess) return e;
    const float* stats = l.stats;
    int64_t from = 0;
    for (int p = 0; p < plan.logits.parts; ++p) {
      const int64_t rows = plan.logits.part[p].rows, parts = div_up(a.n, stat_columns(plan.logits.part[p]));
      k_xent_rows<<<wide_grid(rows), dim3(kRowThreads), 0, stream>>>(a, stats, l.target_z, from, rows, parts);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      from += rows;
      stats += rows * parts * 2;
    }
  }
  if (a.totals) {
    k_xent_totals<<<dim3(1), dim3(1024), 0, stream>>>(a);
    e = hipGetLastError();
  }
  return e;
}

// ---------------------------------------------------------------- gradient
namespace {
// Piece number p: its products, in the order in which they run.
struct Piece {
  LinArgs logits, dx, dw;
};
Piece piece_args(const XentGradArgs& a, int dtype, const XentGradPlan& plan, int64_t p, char* ws) {
  const int64_t bytes = dtype == 1 ? 2 : 4, from = p * plan.width, width = a.n - from < plan.width ? a.n - from : plan.width;
  const char* w = static_cast<const char*>(a.w) + from * a.ldw * bytes;
  void* dz = ws + plan.dz;
  Piece q{};
  q.logits.prod[0] = LinProduct{a.x, w, a.ldx, a.ldw, a.k};
  q.logits.i = a.m;
  q.logits.j = width;
  q.logits.out = dz;
  q.logits.ldout = plan.width;
  q.logits.targets = a.targets;
  q.logits.ignore = a.ignore;
  q.logits.classes = a.n;
  q.logits.col0 = from;
  q.logits.lse = a.lse;
  q.logits.row_scale = a.row_scale;
  q.dx.prod[0] = LinProduct{dz, w, plan.width, a.ldw, width};
  q.dx.i = a.m;
  q.dx.j = a.k;
  q.dx.out = a.dx;
  q.dx.ldout = a.lddx;
  q.dx.ldsum = div_up(a.k, 8) * 8;
  float* sum = reinterpret_cast<float*>(ws + plan.sum);
  q.dx.sum_in = p > 0 ? sum : nullptr;
  q.dx.sum_out = p + 1 < plan.pieces ? sum : nullptr;
  q.dx.scale = a.scale;
  q.dx.totals = a.totals;
  q.dw.prod[0] = LinProduct{dz, a.x, plan.width, a.ldx, a.m};
  q.dw.i = width;
  q.dw.j = a.k;
  q.dw.out = a.dw ? static_cast<char*>(a.dw) + from * a.lddw * bytes : nullptr;
  q.dw.ldout = a.lddw;
  q.dw.scale = a.scale;
  q.dw.totals = a.totals;
  return q;
}
}  // namespace

XentGradPlan xent_grad_plan(const XentGradArgs& a, int dtype) {
  XentGradPlan p{};
  const int64_t bytes = dtype == 1 ? 2 : 4;
  if (a.n == 0 || (!a.dx && !a.dw)) return p;
  // a piece's dz of up to 128 MB stays in the Infinity Cache between the three products that write and read it
  constexpr int64_t kPieceBytes = 128ll << 20, kLeast = 1024;
  int64_t most = a.m > 0 ? kPieceBytes / (a.m * bytes) / 256 * 256 : a.n;
  if (most < kLeast) most = kLeast;
  p.pieces = div_up(a.n, most);
  p.width = div_up(div_up(a.n, p.pieces), 256) * 256;
  p.pieces = div_up(a.n, p.width);
  char* base = reinterpret_cast<char*>(uintptr_t(1) << 20);  // a workspace's address, for its alignment
  for (int last = 0; last < 2; ++last) {
    const Piece q = piece_args(a, dtype, p, last ? p.pieces - 1 : 0, base);
    if (a.m > 0) p.logits[last] = linear_plan(q.logits, dtype, kEpiXentGrad);
    if (a.m > 0 && a.k > 0 && a.dx) p.dx[last] = linear_plan(q.dx, dtype, kEpiSum);
    if (a.k > 0 && a.dw) p.dw[last] = linear_plan(q.dw, dtype, kEpiScaled);
    for (const LinPlan* l : {&p.logits[last], &p.dx[last], &p.dw[last]})
      if (l->workspace > p.product) p.product = l->workspace;
  }
  p.dz = round16(p.product);
  p.sum = p.dz + round16((size_t)a.m * (size_t)p.width * (size_t)bytes);
  p.workspace = p.sum + (a.dx && p.pieces > 1 ? (size_t)a.m * (size_t)(div_up(a.k, 8) * 8) * 4 : 0);
  return p;
}

hipError_t launch_xent_grad(const XentGradArgs& a, int dtype, const XentGradPlan& plan, void* workspace, hipStream_t stream) {
  hipError_t e = hipSuccess;
  for (int64_t p = 0; p < plan.pieces; ++p) {
    const Piece q = piece_args(a, dtype, plan, p, static_cast<char*>(workspace));
    const int last = p + 1 == plan.pieces;
    if (a.m > 0) e = launch_linear(q.logits, dtype, kEpiXentGrad, plan.logits[last], workspace, stream);
    if (e == hipSuccess && a.m > 0 && a.k > 0 && a.dx) e = launch_linear(q.dx, dtype, kEpiSum, plan.dx[last], workspace, stream);
    if (e == hipSuccess && a.k > 0 && a.dw) e = launch_linear(q.dw, dtype, kEpiScaled, plan.dw[last], workspace, stream);
    if (e != hipSuccess) break;
  }
  return e;
}

}  // namespace smat
