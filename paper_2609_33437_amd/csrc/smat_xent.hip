// The output layer with its cross entropy for gfx950: z = x W^T over a vocabulary, without keeping z.
//
//   lse_i = log sum_j exp z_ij,  loss_i = lse_i - z_i,t_i
//   dz_ij = (exp(z_ij - lse_i) - [j = t_i]) g_i,  dx = s dz W,  dW = s dz^T x
//
// lse is the largest logit plus a log between 0 and log n, and where logits are in the hundreds its rounding to fp32 exceeds
// 1 - p of a target that has nearly the whole probability.  So it is held as two fp32 numbers, and p - 1 is an expm1 of
// their difference from the logit: such a row's dz keeps its digits down to 1 - p of 2^-24, and sums to 0.
//
// The forward product's epilogue leaves the largest value and the sum of exponentials of each tile's columns of a row, which
// k_xent_rows joins.  The gradient goes through the vocabulary in pieces: a piece's logits again, turned into dz (in the
// call's dtype) by their epilogue, then dz W added to dx in fp32 and dz^T x, which is the piece's part of dW.  So beside
// its outputs a call holds one piece of dz, a copy of x and, with several pieces, fp32 sums of dx, whatever the vocabulary, for a
// fourth product beside the three that cannot be left out.  s is applied to the fp32 sums of both products, so a mean over many rows costs dz no precision.
#include "smat_decoder.h"
#include "smat_linear_dev.h"

namespace smat {
namespace {

constexpr int kRowThreads = 256;

// A row's log sum of exponentials from its parts, and its loss.  Eight parts a thread are loaded together (1 row of 50304 / 32
// parts: 3.9 us, 4.8 one by one).
__global__ __launch_bounds__(kRowThreads) void k_xent_rows(XentArgs a, const float* stats, const float* target_z, int64_t from,
                                                           int64_t rows, int64_t parts) {
  constexpr int kAhead = 8;
  __shared__ float tops[kRowThreads / 64], sums[kRowThreads / 64];
  if (wide_block() >= rows) return;
  const f32x2* s = reinterpret_cast<const f32x2*>(stats) + wide_block() * parts;
  const int64_t i = from + wide_block();
  float top = -__builtin_inff(), sum = 0.f;
  for (int64_t k0 = 0; k0 < parts; k0 += kAhead * kRowThreads) {
    f32x2 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t k = k0 + u * kRowThreads + threadIdx.x;
      v[u] = f32x2{-__builtin_inff(), 0.f};
      if (k < parts) v[u] = s[k];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (k0 + u * kRowThreads < parts) join_stats(top, sum, v[u][0], v[u][1]);
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
  const float rest = logf(sum);
  const int64_t t = a.targets[i];
  const float lse = rest + top;
  a.lse[i] = lse;
  if (a.lse_low) {  // what the sum's rounding left, exactly
    const float part = lse - top;
    a.lse_low[i] = __builtin_isfinite(lse) ? (top - (lse - part)) + (rest - part) : 0.f;
  }
  // from the largest value on, not from lse, whose rounding may be larger than a small loss
  a.loss[i] = t == a.ignore ? 0.f : t < 0 || t >= a.n ? __builtin_nanf("") : rest + (top - target_z[i]);
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

// ---------------------------------------------------------------- rows with a target
namespace {
// The rows whose target is not the one to ignore, in order: theirs of the vectors, where they came from, how many (and how
// many among the logits' first rows), and each row's place among them (-1: none).
struct SomeRows {
  int64_t* targets;
  float* lse;
  float* lse_low;
  float* row_scale;
  int32_t* from;
  int32_t* place;
  int32_t* count;
};
SomeRows some_rows(char* at, int64_t m) {
  SomeRows r{};
  r.targets = reinterpret_cast<int64_t*>(at);
  r.lse = reinterpret_cast<float*>(r.targets + m);
  r.lse_low = r.lse + m;
  r.row_scale = r.lse_low + m;
  r.from = reinterpret_cast<int32_t*>(r.row_scale + m);
  r.place = r.from + m;
  r.count = r.place + m;
  return r;
}
constexpr int64_t some_rows_bytes(int64_t m) { return m * 28 + 8; }

__global__ __launch_bounds__(1024) void k_xent_some(XentGradArgs a, SomeRows r, int64_t first) {
  __shared__ int32_t waves[2][16];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  int32_t before = 0;
  int parity = 0;
  for (int64_t i0 = 0; i0 < a.m; i0 += 1024, parity ^= 1) {
    const int64_t i = i0 + threadIdx.x;
    const int64_t t = i < a.m ? a.targets[i] : a.ignore;
    const bool on = t != a.ignore;
    const uint64_t all = __ballot(on);
    if (lane == 0) waves[parity][wave] = __popcll(all);
    __syncthreads();
    int32_t at = before + __popcll(all & ((uint64_t(1) << lane) - 1));
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      at += k < wave ? waves[parity][k] : 0;
      before += waves[parity][k];
    }
    if (i == first) r.count[1] = at;
    if (i < a.m) r.place[i] = on ? at : -1;
    if (on) {
      r.from[at] = (int32_t)i;
      r.targets[at] = t;
      r.lse[at] = a.lse[i];
      if (a.lse_low) r.lse_low[at] = a.lse_low[i];
      if (a.row_scale) r.row_scale[at] = a.row_scale[i];
    }
  }
  if (threadIdx.x == 0) *r.count = before;
}

// x on 16-byte rows with zeros at their ends, a wave a row: rows without a target as zeros, so that a padded row's NaN
// reaches no gradient, or with `place` the other rows alone, and then the zeros of such rows of dx too.
template <typename T>
__global__ __launch_bounds__(256) void k_xent_rows_of_x(XentGradArgs a, const int32_t* place, void* to, int64_t stride) {
  using Mem = typename El<T>::Mem;
  const int64_t i = wide_block() * 4 + ((int)threadIdx.x >> 6), first = (int64_t)(threadIdx.x & 63) * 8;
  if (i >= a.m) return;
  const int64_t at = place ? place[i] : i;
  const bool on = place ? at >= 0 : a.targets[i] != a.ignore;
  const float zeros[8] = {};
  if (at >= 0) {
    const Mem* x = static_cast<const Mem*>(a.x) + i * a.ldx;
    Mem* row = static_cast<Mem*>(to) + at * stride;
#pragma unroll 4
    for (int64_t j = first; j < stride; j += 512) {
      float v[8];
      load_row8<T>(x + j, on ? a.k - j : 0, v);
      store_row8<T>(row + j, stride - j, v);
    }
  } else if (a.dx) {
    Mem* row = static_cast<Mem*>(a.dx) + i * a.lddx;
#pragma unroll 4
    for (int64_t j = first; j < a.k; j += 512) store_row8<T>(row + j, a.k - j, zeros);
  }
}
}  // namespace

// ---------------------------------------------------------------- gradient
namespace {
// Piece number p: its products, in the order in which they run.
struct Piece {
  LinArgs logits, dx, dw;
};
Piece piece_args(const XentGradArgs& a, int dtype, const XentGradPlan& plan, int64_t p, char* ws) {
  const int64_t bytes = dtype == 1 ? 2 : 4, from = p * plan.width, width = a.n - from < plan.width ? a.n - from : plan.width;
  const int64_t packed = packed_stride(a.k, dtype);
  const void* w = static_cast<const char*>(a.w) + from * a.ldw * bytes;
  const void* x = ws + plan.x;
  const int64_t ldx = packed;
  int64_t ldw = a.ldw;
  if (plan.pack) {
    w = ws + plan.w;
    ldw = packed;
  }
  char *dz = ws + plan.dz, *low = plan.low ? dz + a.m * plan.width * bytes : nullptr;
  Piece q{};
  q.logits.prod[0] = LinProduct{x, w, ldx, ldw, plan.pack ? packed : a.k};  // both end in zeros
  q.logits.i = a.m;
  q.logits.j = width;
  q.logits.out = dz;
  q.logits.ldout = plan.width;
  q.logits.out_low = low;
  q.logits.targets = a.targets;
  q.logits.ignore = a.ignore;
  q.logits.classes = a.n;
  q.logits.col0 = from;
  q.logits.lse = a.lse;
  q.logits.lse_low = a.lse_low;
  q.logits.row_scale = a.row_scale;
  q.dx.prod[0] = LinProduct{dz, w, plan.width, ldw, width};
  if (low) q.dx.prod[1] = LinProduct{low, w, plan.width, ldw, width};
  q.dx.p_clean = 1;
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
  if (plan.some) {
    const SomeRows r = some_rows(ws + plan.rows, a.m);
    q.logits.targets = r.targets;
    q.logits.lse = r.lse;
    if (a.lse_low) q.logits.lse_low = r.lse_low;
    if (a.row_scale) q.logits.row_scale = r.row_scale;
    q.dx.out_rows = r.from;
    q.logits.count = q.dx.count = q.dw.count = r.count;
    if (plan.first) q.logits.first_count = r.count + 1;
  } else {
    q.dx.targets = a.targets;
    q.dx.ignore = a.ignore;
  }
  q.dw.prod[0] = LinProduct{dz, x, plan.width, ldx, a.m};
  if (low) q.dw.prod[1] = LinProduct{low, x, plan.width, ldx, a.m};
  q.dw.i = width;
  q.dw.j = a.k;
  q.dw.out = a.dw ? static_cast<char*>(a.dw) + from * a.lddw * bytes : nullptr;
  q.dw.ldout = a.lddw;
  q.dw.scale = a.scale;
  q.dw.totals = a.totals;
  return q;
}

bool on_16_bytes(const void* p, int64_t ld, int64_t run, int64_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * bytes % 16 == 0 && run * bytes % 16 == 0;
}

constexpr int64_t kLowRows = 128;

// The products' plans and the workspace where x and W are copied as `pack` says; their estimated microseconds.
double plan_products(const XentGradArgs& a, int dtype, XentGradPlan& p, const LinPlan* like) {
  const int64_t bytes = dtype == 1 ? 2 : 4;
  char* base = reinterpret_cast<char*>(uintptr_t(1) << 20);  // a workspace's address, for its alignment
  double us = 0.0;
  size_t product = 0;
  p.dz = p.sum = p.x = p.w = p.rows = 0;
  for (int last = 0; last < 2; ++last) {
    const Piece q = piece_args(a, dtype, p, last ? p.pieces - 1 : 0, base);
    p.logits[last] = p.dx[last] = p.dw[last] = LinPlan{};
    if (a.m > 0) p.logits[last] = linear_plan(q.logits, dtype, kEpiXentGrad, like);
    if (a.m > 0 && a.k > 0 && a.dx) p.dx[last] = linear_plan(q.dx, dtype, kEpiSum);
    if (a.k > 0 && a.dw) p.dw[last] = linear_plan(q.dw, dtype, kEpiScaled);
    double piece = 0.0;
    for (const LinPlan* l : {&p.logits[last], &p.dx[last], &p.dw[last]}) {
      if (l->workspace > product) product = l->workspace;
      // bf16 stages by way of registers take up to 1.5 times their estimate, which decides between them and a copy of W.  Calls
      // copied and by way of registers, where the factor makes the choice: 33 x 62106 x 1537 361 and 456 us, 160 x 62106 x 4097
      // 850 and 896, 300 x 10007 x 2982 138 and 146, 160 x 32003 x 1537 209 and 207, 9 x 62106 x 769 195 and 178, 100 x 62106 x 2982
      // 633 and 545: over 15 sizes the copies spare up to 26 % and cost up to 14 %
      piece += l->us * (dtype == 1 && l->parts && !l->direct ? 1.5 : 1.0);
    }
    if (p.pack) piece += pack_us((double)q.logits.j * (double)a.k * (double)bytes);
    us += piece * (double)(last ? 1 : p.pieces - 1);
  }
  size_t at = round16(product);
  const auto take = [&](int64_t elements, int64_t size, bool wanted) {
    const size_t here = at;
    if (wanted) at += round16((size_t)elements * (size_t)size);
    return here;
  };
  const int64_t packed = packed_stride(a.k, dtype);
  p.dz = take(a.m * p.width * (p.low ? 2 : 1), bytes, true);
  p.sum = take(a.m * (div_up(a.k, 8) * 8), 4, a.dx && p.pieces > 1);
  p.x = take(a.m * packed, bytes, true);
  p.w = take(p.width * packed, bytes, p.pack);
  p.rows = take(some_rows_bytes(a.m), 1, p.some);
  p.workspace = at;
  return us;
}
}  // namespace

XentGradPlan xent_grad_plan(const XentGradArgs& a, int dtype) {
  XentGradPlan p{};
  const int64_t bytes = dtype == 1 ? 2 : 4;
  if (!a.dx && !a.dw) return p;
  // With both halves of dz multiplied, dx and dW are as exact as their own rounding; with one, theirs and dz's add up.  Up to
  // kLowRows rows, where W's and dW's bytes bound the products, the second half costs a quarter or a third (32000 x 1024: 32 rows 77 us
  // and 62, errors of dx and dW against float64 1.66e-3 and 1.43e-3 of their norms, 2.07e-3 and 1.90e-3; 128 rows 99 us and 75,
  // 1.66e-3 and 1.38e-3, 2.01e-3 and 1.74e-3), with more up to a half (512 rows 205 us and 140, 1.66e-3 and 1.47e-3, 1.97e-3 and
  // 1.81e-3).
  p.low = dtype == 1 && a.m <= kLowRows;
  // a piece's dz of about 128 MB stays in the Infinity Cache between the three products that write and read it
  // (4096 x 128256 x 2048: 6.61 ms with losses, in pieces of 64 MB 6.81 ms, of 512 MB 6.53 ms, in one of 1.05 GB 6.50 ms)
  constexpr int64_t kPieceBytes = 128ll << 20, kLeast = 1024;
  int64_t most = a.m > 0 ? kPieceBytes / (a.m * bytes) / 256 * 256 : a.n;
  if (most < kLeast) most = kLeast;
  p.pieces = div_up(a.n, most);
  p.width = div_up(div_up(a.n, p.pieces), 256) * 256;
  p.pieces = div_up(a.n, p.width);
  // the choices below are those for both gradients, so that each has the same bits when it is wanted alone
  XentGradArgs both = a;
  if (!a.dx) both.dx = a.dw;
  if (!a.dw) both.dw = a.dx;
  // The logits' sums take the order of the losses' call.  What a logit lost there to rounding is in the log sum too, so
  // exp(z - lse) of a probable class is exact; by sums in another order it is off by both logits' (fp32 157 x 43584 x 2829: dW by
  // 3.3e-6 of its norm, by 1.1e-6 so; bf16 2100 x 60000 x 2048 with targets of logit 600 and probability 1: dx, which is 0, up to
  // 1.7e-3 in the 52 rows left over for another tile).
  LinPlan losses{};
  if (a.m > 0) losses = xent_plan(XentArgs{a.x, a.w, a.ldx, a.ldw, a.m, a.n, a.k}, dtype).logits;
  const LinPlan* like = losses.parts ? &losses : nullptr;
  double us = plan_products(both, dtype, p, like);
  // rows of W off 16 bytes serve two products: a copy of each piece for both, where that is estimated to be faster
  if (a.m > 0 && a.k > 0 && !on_16_bytes(a.w, a.ldw, a.k, bytes)) {
    XentGradPlan q = p;
    q.pack = 1;
    const double copied = plan_products(both, dtype, q, like);
    if (copied < us) {
      us = copied;
      p = q;
    }
  }
  // Rows without a target (a prompt's, padding) have no gradient.  Only the device knows them, so the launches are for all rows
  // and blocks without any end at once.  A launch finds them; it is spent where it is estimated at a fiftieth of the call or
  // less.  (2048 x 128256 x 4096, half of the rows without: losses and gradients 4.75 ms, 6.15 ms with
  // products over all rows.)
  p.some = a.m > 0 && a.k > 0 && !p.low && us > 50.0 * (10.0 + (double)a.m / 1000.0);
  plan_products(a, dtype, p, like);
  // A row left out moves the ones behind it up, but not into a part that sums in another order than theirs (fp32 515 x 32003 x 769
  // with a tenth of the rows without a target: 765 us; 742 where the 464 rows leave none to the second part, whose rows then
  // have logits other than their log sum's).
  if (p.some && like && !one_order(*like)) {
    const int64_t rows = like->part[0].rows;
    if (p.logits[0].parts == 2 && p.logits[0].part[0].rows == rows && p.logits[1].parts == 2 && p.logits[1].part[0].rows == rows) p.first = rows;
  }
  return p;
}

hipError_t launch_xent_grad(const XentGradArgs& a, int dtype, const XentGradPlan& plan, void* workspace, hipStream_t stream) {
  hipError_t e = hipSuccess;
  char* ws = static_cast<char*>(workspace);
  if (plan.pieces == 0) return e;  // no gradient is wanted, and there is no workspace
  if (a.m > 0) {
    const int32_t* place = nullptr;
    if (plan.some) {
      const SomeRows r = some_rows(ws + plan.rows, a.m);
      k_xent_some<<<dim3(1), dim3(1024), 0, stream>>>(a, r, plan.first);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      place = r.place;
    }
    const dim3 grid = wide_grid(div_up(a.m, 4));
    if (dtype == 1)
      k_xent_rows_of_x<Bf16><<<grid, dim3(256), 0, stream>>>(a, place, ws + plan.x, packed_stride(a.k, dtype));
    else
      k_xent_rows_of_x<float><<<grid, dim3(256), 0, stream>>>(a, place, ws + plan.x, packed_stride(a.k, dtype));
    e = hipGetLastError();
  }
  for (int64_t p = 0; p < plan.pieces && e == hipSuccess; ++p) {
    const Piece q = piece_args(a, dtype, plan, p, ws);
    const int last = p + 1 == plan.pieces;
    if (plan.pack) {
      const char* w = static_cast<const char*>(a.w) + p * plan.width * a.ldw * (dtype == 1 ? 2 : 4);
      if ((e = launch_pack(w, a.ldw, q.logits.j, a.k, dtype, ws + plan.w, stream)) != hipSuccess) break;
    }
    if (a.m > 0) e = launch_linear(q.logits, dtype, kEpiXentGrad, plan.logits[last], workspace, stream);
    if (e == hipSuccess && a.m > 0 && a.k > 0 && a.dx) e = launch_linear(q.dx, dtype, kEpiSum, plan.dx[last], workspace, stream);
    if (e == hipSuccess && a.k > 0 && a.dw) e = launch_linear(q.dw, dtype, kEpiScaled, plan.dw[last], workspace, stream);
  }
  return e;
}

}  // namespace smat
