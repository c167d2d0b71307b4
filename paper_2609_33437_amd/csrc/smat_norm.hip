// Norms over the rows of a matrix for gfx950, forward and backward.
//
//   layer  mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) r, y = xh w + b
//   rms    mu = 0
//   dx = r (g - xh mean(g xh) - mean(g)) with g = dy w (rms: without mean(g)), dw = sum_rows dy xh, db = sum_rows dy
//
// Bound by HBM: the forward pass reads and writes a row once, the backward reads two and writes one: 16384 x 4096 bf16 takes
// 44 us, 6.1 TB/s, and 79 us, 5.1 TB/s, with 5 us more to join the blocks' sums.  A row is held in
// registers between its sums and its use, by 16 to 1024 threads with one or two eights of columns each, so the variance is
// the sum of squared differences from the mean, not a difference of sums.  Statistics and sums are fp32.
#include "smat_decoder.h"
#include "smat_linear_dev.h"

namespace smat {
namespace {

// `threads` of a block share a row and hold E eights of it each.  AHEAD: the next row's loads are under way while a row is
// used (16384 x 4096 bf16 backward: 81 us, 130 us without); two eights in each of 1024 threads have no registers for it.
template <int THREADS, int E, bool AHEAD = true>
struct RowShape {
  static constexpr bool kAhead = AHEAD;
  static constexpr int kThreads = THREADS, kE = E;
  static constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kRows = kBlock / THREADS, kColumns = THREADS * E * 8;
};
constexpr int64_t kMaxHeld = 1024 * 2 * 8;  // columns of the widest shape

// Eight weights of either type, ones or zeros where there are none.
__device__ __forceinline__ void load_weights(const void* w, int dtype, int64_t j, int64_t valid, float none, float v[8]) {
  if (!w || valid <= 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = none;
  } else if (dtype == SMAT_BF16) {
    load_row8<Bf16>(static_cast<const uint16_t*>(w) + j, valid, v);
  } else {
    load_row8<float>(static_cast<const float*>(w) + j, valid, v);
  }
}
__device__ __forceinline__ void store_weight(void* w, int dtype, int64_t j, float v) {
  if (dtype == SMAT_BF16)
    El<Bf16>::store(static_cast<uint16_t*>(w) + j, v);
  else
    static_cast<float*>(w)[j] = v;
}

// Sums of N values over the threads of a row.  `slot` is LDS of N floats a wave that nothing else uses until every thread
// has passed another of these calls.
template <int THREADS, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum<(THREADS < 64 ? THREADS : 64)>(v[i]);
  if constexpr (THREADS > 64) {
    constexpr int kWaves = THREADS / 64;
    const int wave = (int)threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) slot[i * kWaves + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) v[i] += slot[i * kWaves + k];
    }
  }
}

// A row's eights of one matrix as they lie in memory, loaded ahead of their use.
template <typename T, typename S>
struct RowRaw {
  Raw8<T> x[S::kE];
  __device__ __forceinline__ void load(const typename El<T>::Mem* row, int64_t n, int lane) {
#pragma unroll
    for (int e = 0; e < S::kE; ++e) {
      const int64_t j = (int64_t)(e * S::kThreads + lane) * 8;
      x[e].load_some(row + j, n - j);
    }
  }
};

// Blocks take rows in turn; the next row's loads are under way while a row is summed and stored.
template <typename T, typename S>
__global__ __launch_bounds__(S::kBlock) void k_norm(NormArgs a) {
  using Mem = typename El<T>::Mem;
  constexpr int kWaves = S::kThreads > 64 ? S::kThreads / 64 : 1;
  __shared__ float slots[4][kWaves];
  const int lane = (int)threadIdx.x % S::kThreads;
  const Mem* x = static_cast<const Mem*>(a.x);
  const int64_t step = (int64_t)gridDim.x * S::kRows;
  int64_t row = (int64_t)blockIdx.x * S::kRows + (int)threadIdx.x / S::kThreads;
  if (row >= a.m) return;  // whole rows of threads, and whole blocks where they share LDS
  RowRaw<T, S> raw;
  raw.load(x + row * a.ldx, a.n, lane);
  float w[S::kE][8], b[S::kE][8];
#pragma unroll
  for (int e = 0; e < S::kE; ++e) {
    const int64_t j = (int64_t)(e * S::kThreads + lane) * 8;
    load_weights(a.w, a.wdtype, j, a.n - j, 1.f, w[e]);
    load_weights(a.b, a.wdtype, j, a.n - j, 0.f, b[e]);
  }
  const float inverse = 1.f / (float)a.n;
  for (int parity = 0; row < a.m; row += step, parity ^= 2) {
    float v[S::kE][8];
#pragma unroll
    for (int e = 0; e < S::kE; ++e) raw.x[e].get(v[e]);
    if (S::kAhead && row + step < a.m) raw.load(x + (row + step) * a.ldx, a.n, lane);
    float mu = 0.f;
    if (a.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < S::kE; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += v[e][i];
      row_sums<S::kThreads>(s, slots[parity]);
      mu = s[0] * inverse;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < S::kE; ++e) {
      const int64_t valid = a.n - (int64_t)(e * S::kThreads + lane) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[e][i] = i < valid ? v[e][i] - mu : 0.f;
        s[0] = __builtin_fmaf(v[e][i], v[e][i], s[0]);
      }
    }
    row_sums<S::kThreads>(s, slots[parity + 1]);
    const float r = 1.f / sqrtf(s[0] * inverse + a.eps);
    if (lane == 0) {
      if (a.mean) a.mean[row] = mu;
      if (a.rstd) a.rstd[row] = r;
    }
    Mem* y = static_cast<Mem*>(a.y) + row * a.ldy;
#pragma unroll
    for (int e = 0; e < S::kE; ++e) {
      const int64_t j = (int64_t)(e * S::kThreads + lane) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[e][i] = __builtin_fmaf(v[e][i] * r, w[e][i], b[e][i]);
      store_row8<T>(y + j, a.n - j, v[e]);
    }
    if (!S::kAhead && row + step < a.m) raw.load(x + (row + step) * a.ldx, a.n, lane);
  }
}

// Rows too wide for registers: three reads of a row by one block.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_wide(NormArgs a) {
  using Mem = typename El<T>::Mem;
  __shared__ float slots[2][16];
  const int64_t row = wide_block();
  if (row >= a.m) return;
  const Mem* x = static_cast<const Mem*>(a.x) + row * a.ldx;
  Mem* y = static_cast<Mem*>(a.y) + row * a.ldy;
  const float inverse = 1.f / (float)a.n;
  float mu = 0.f;
  if (a.layer) {
    float s[1] = {0.f};
    for (int64_t j = (int64_t)threadIdx.x * 8; j < a.n; j += 8192) {
      float v[8];
      load_row8<T>(x + j, a.n - j, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[i];
    }
    row_sums<1024>(s, slots[0]);
    mu = s[0] * inverse;
  }
  float s[1] = {0.f};
  for (int64_t j = (int64_t)threadIdx.x * 8; j < a.n; j += 8192) {
    float v[8];
    load_row8<T>(x + j, a.n - j, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = j + i < a.n ? v[i] - mu : 0.f;
      s[0] = __builtin_fmaf(d, d, s[0]);
    }
  }
  row_sums<1024>(s, slots[1]);
  const float r = 1.f / sqrtf(s[0] * inverse + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
  for (int64_t j = (int64_t)threadIdx.x * 8; j < a.n; j += 8192) {
    float v[8], w[8], b[8];
    load_row8<T>(x + j, a.n - j, v);
    load_weights(a.w, a.wdtype, j, a.n - j, 1.f, w);
    load_weights(a.b, a.wdtype, j, a.n - j, 0.f, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf((v[i] - mu) * r, w[i], b[i]);
    store_row8<T>(y + j, a.n - j, v);
  }
}

// Blocks take rows in turn and keep their sums of dw and db in registers; k_norm_join adds the blocks' sums in order.
template <typename T, typename S>
__global__ __launch_bounds__(S::kBlock) void k_norm_grad(NormGradArgs a) {
  using Mem = typename El<T>::Mem;
  constexpr int kWaves = S::kThreads > 64 ? S::kThreads / 64 : 1;
  __shared__ float slots[2][2 * kWaves];
  __shared__ float shared[S::kRows > 1 ? S::kColumns : 1];
  const int lane = (int)threadIdx.x % S::kThreads, group = (int)threadIdx.x / S::kThreads;
  float w[S::kE][8], dw[S::kE][8] = {}, db[S::kE][8] = {};
  const auto load_w = [&] {
#pragma unroll
    for (int e = 0; e < S::kE; ++e) {
      const int64_t j = (int64_t)(e * S::kThreads + lane) * 8;
      load_weights(a.w, a.wdtype, j, a.n - j, 1.f, w[e]);
    }
  };
  if (S::kAhead) load_w();
  const float inverse = 1.f / (float)a.n;
  int parity = 0;
  const Mem *x = static_cast<const Mem*>(a.x), *dy = static_cast<const Mem*>(a.dy);
  const int64_t step = (int64_t)gridDim.x * S::kRows;
  int64_t row = (int64_t)blockIdx.x * S::kRows + group;
  RowRaw<T, S> raw_x, raw_dy;
  float next_mu = 0.f, next_r = 0.f;
  const auto load = [&](int64_t i) {
    raw_x.load(x + i * a.ldx, a.n, lane);
    raw_dy.load(dy + i * a.lddy, a.n, lane);
    if (a.layer) next_mu = a.mean[i];
    next_r = a.rstd[i];
  };
  if (row < a.m) load(row);
  for (; row < a.m; row += step) {
    float xh[S::kE][8], g[S::kE][8];
#pragma unroll
    for (int e = 0; e < S::kE; ++e) {
      raw_x.x[e].get(xh[e]);
      raw_dy.x[e].get(g[e]);
    }
    const float mu = next_mu, r = next_r;
    if (!S::kAhead) load_w();
    if (S::kAhead && row + step < a.m) load(row + step);
    float s[2] = {0.f, 0.f};  // of g xh and g
#pragma unroll
    for (int e = 0; e < S::kE; ++e) {
      const int64_t valid = a.n - (int64_t)(e * S::kThreads + lane) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xh[e][i] = i < valid ? (xh[e][i] - mu) * r : 0.f;
        dw[e][i] = __builtin_fmaf(g[e][i], xh[e][i], dw[e][i]);
        db[e][i] += g[e][i];
        g[e][i] *= w[e][i];
        s[0] = __builtin_fmaf(g[e][i], xh[e][i], s[0]);
        s[1] += g[e][i];
      }
    }
    if (a.dx) {
      row_sums<S::kThreads>(s, slots[parity]);
      parity ^= 1;
      const float along = s[0] * inverse, mean = a.layer ? s[1] * inverse : 0.f;
      Mem* dx = static_cast<Mem*>(a.dx) + row * a.lddx;
#pragma unroll
      for (int e = 0; e < S::kE; ++e) {
        const int64_t j = (int64_t)(e * S::kThreads + lane) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) g[e][i] = r * (__builtin_fmaf(-xh[e][i], along, g[e][i]) - mean);
        store_row8<T>(dx + j, a.n - j, g[e]);
      }
    }
    if (!S::kAhead && row + step < a.m) load(row + step);
  }
  // the block's sums, its groups' added in order
  for (int which = 0; which < 2; ++which) {
    if (!(which ? a.db : a.dw)) continue;
    void* last = which ? a.db : a.dw;  // of one block
    float* to = a.partial + ((int64_t)(which && a.dw ? a.blocks : 0) + blockIdx.x) * a.n;
    if constexpr (S::kRows > 1) {
      for (int k = 0; k < S::kRows; ++k) {
        __syncthreads();
        if (group == k) {
#pragma unroll
          for (int e = 0; e < S::kE; ++e)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              // one bank for each lane: column i of eight number c lies at i * eights + c
              float* p = shared + i * (S::kColumns / 8) + e * S::kThreads + lane;
              const float v = which ? db[e][i] : dw[e][i];
              *p = k ? *p + v : v;
            }
        }
      }
      __syncthreads();
      for (int j = (int)threadIdx.x; j < a.n; j += S::kBlock) {
        const float v = shared[j % 8 * (S::kColumns / 8) + j / 8];
        if (a.blocks == 1)
          store_weight(last, a.wdtype, j, v);
        else
          to[j] = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < S::kE; ++e) {
        const int64_t j = (int64_t)(e * S::kThreads + lane) * 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = which ? db[e][i] : dw[e][i];
        if (a.blocks > 1)
          store_row8<float>(to + j, a.n - j, v);
        else if (a.wdtype == SMAT_BF16)
          store_row8<Bf16>(static_cast<uint16_t*>(last) + j, a.n - j, v);
        else
          store_row8<float>(static_cast<float*>(last) + j, a.n - j, v);
      }
    }
  }
}

// Rows too wide for registers: dx by a block a row, which reads x and dy twice.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_grad_wide(NormGradArgs a) {
  using Mem = typename El<T>::Mem;
  __shared__ float slots[32];
  const int64_t row = wide_block();
  if (row >= a.m) return;
  const Mem* x = static_cast<const Mem*>(a.x) + row * a.ldx;
  const Mem* dy = static_cast<const Mem*>(a.dy) + row * a.lddy;
  Mem* dx = static_cast<Mem*>(a.dx) + row * a.lddx;
  const float mu = a.layer ? a.mean[row] : 0.f, r = a.rstd[row], inverse = 1.f / (float)a.n;
  const auto load = [&](int64_t j, float xh[8], float g[8]) {
    float w[8];
    load_row8<T>(x + j, a.n - j, xh);
    load_row8<T>(dy + j, a.n - j, g);
    load_weights(a.w, a.wdtype, j, a.n - j, 1.f, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      xh[i] = j + i < a.n ? (xh[i] - mu) * r : 0.f;
      g[i] *= w[i];
    }
  };
  float s[2] = {0.f, 0.f};
  for (int64_t j = (int64_t)threadIdx.x * 8; j < a.n; j += 8192) {
    float xh[8], g[8];
    load(j, xh, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[0] = __builtin_fmaf(g[i], xh[i], s[0]);
      s[1] += g[i];
    }
  }
  row_sums<1024>(s, slots);
  const float along = s[0] * inverse, mean = a.layer ? s[1] * inverse : 0.f;
  for (int64_t j = (int64_t)threadIdx.x * 8; j < a.n; j += 8192) {
    float xh[8], g[8];
    load(j, xh, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = r * (__builtin_fmaf(-xh[i], along, g[i]) - mean);
    store_row8<T>(dx + j, a.n - j, g);
  }
}

// Their sums of dw and db: a thread takes eight columns of every blocks-th row.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_columns_wide(NormGradArgs a) {
  using Mem = typename El<T>::Mem;
  const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (j >= a.n) return;
  float dw[8] = {}, db[8] = {};
  for (int64_t row = blockIdx.y; row < a.m; row += a.blocks) {
    float x[8], dy[8];
    load_row8<T>(static_cast<const Mem*>(a.x) + row * a.ldx + j, a.n - j, x);
    load_row8<T>(static_cast<const Mem*>(a.dy) + row * a.lddy + j, a.n - j, dy);
    const float mu = a.layer ? a.mean[row] : 0.f, r = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dw[i] = __builtin_fmaf(dy[i], (x[i] - mu) * r, dw[i]);
      db[i] += dy[i];
    }
  }
  if (a.dw) store_row8<float>(a.partial + (int64_t)blockIdx.y * a.n + j, a.n - j, dw);
  if (a.db) store_row8<float>(a.partial + ((int64_t)(a.dw ? a.blocks : 0) + blockIdx.y) * a.n + j, a.n - j, db);
}

// dw (blockIdx.z = 0) and db as the sums of the blocks' sums: 32 columns a block, 32 groups of rows, added in order.
constexpr int kJoinColumns = 32, kJoinRows = 32;
__global__ __launch_bounds__(kJoinColumns* kJoinRows) void k_norm_join(NormGradArgs a) {
  __shared__ float s[kJoinRows][kJoinColumns + 1];
  const int c = (int)threadIdx.x % kJoinColumns, g = (int)threadIdx.x / kJoinColumns;
  const int64_t j = wide_block() * kJoinColumns + c;
  const bool second = blockIdx.z != 0 || !a.dw;
  const float* from = a.partial + (int64_t)(blockIdx.z ? a.blocks : 0) * a.n;
  float sum = 0.f;
  if (j < a.n) {
#pragma unroll 8
    for (int32_t k = g; k < a.blocks; k += kJoinRows) sum += from[(int64_t)k * a.n + j];
  }
  s[g][c] = sum;
  __syncthreads();
  if (g == 0 && j < a.n) {
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k) sum += s[k][c];
    store_weight(second ? a.db : a.dw, a.wdtype, j, sum);
  }
}

// ---------------------------------------------------------------- launches
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
template <typename F>
void with_element(int dtype, F&& fn) {
  if (dtype == 1)
    fn(Bf16());
  else
    fn(float());
}

// fn(shape) for rows of n <= kMaxHeld columns: few threads, whose sums cost least, as long as their registers let enough of
// them be resident (12115 x 5544 with 1024 threads of one eight 55 and 83 us, with 512 of two 43 and 82, with 256 of four, without
// loads ahead, 48 and 136).
template <typename F>
void with_shape(int64_t n, F&& fn) {
  if (n <= 128)
    fn(RowShape<16, 1>());
  else if (n <= 512)
    fn(RowShape<64, 1>());
  else if (n <= 1024)
    fn(RowShape<64, 2>());
  else if (n <= 2048)
    fn(RowShape<256, 1>());
  else if (n <= 4096)
    fn(RowShape<256, 2>());
  else if (n <= 8192)
    fn(RowShape<512, 2>());
  else
    fn(RowShape<1024, 2, false>());
}
}  // namespace

hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t stream) {
  with_element(dtype, [&](auto t) {
    using T = decltype(t);
    if (a.n > kMaxHeld) {
      k_norm_wide<T><<<wide_grid(a.m), dim3(1024), 0, stream>>>(a);
      return;
    }
    with_shape(a.n, [&](auto s) {
      using S = decltype(s);
      // 4096 blocks of 256 threads, several times what is resident, so that the last ones are spread; one row a block takes 53 us
      // for 16384 x 4096, these 44
      const int64_t blocks = div_up(a.m, S::kRows), most = 16 * 256 / (S::kBlock / 256);
      k_norm<T, S><<<dim3((uint32_t)(blocks < most ? blocks : most)), dim3(S::kBlock), 0, stream>>>(a);
    });
  });
  return hipGetLastError();
}

int32_t norm_grad_blocks(int64_t m, int64_t n) {
  int64_t rows = 1;
  if (n <= kMaxHeld) with_shape(n, [&](auto s) { rows = decltype(s)::kRows; });
  const int64_t blocks = div_up(m, rows);
  // a handful of rows is one block's, which writes dw and db itself and spares the second launch. Replayed, two rows of 4096 take
  // 4.8 us so and 6.1 apart, of 16384 10.7 and 11.8; three 5.8 and 6.1, 13.3 and 11.8. A call with 8 x 64 takes 9.0 us, host
  // bound, and 13.2 with two launches.
  if (n <= kMaxHeld && blocks > 0 && blocks <= 2) return 1;
  // One block a compute unit; two where rows are narrow and each block still has several turns.  Replayed on rows that are not in a
  // cache, with the join, 256 and 512 blocks: 600 x 4096 14.3 and 18.1 us, 1024 x 2048 11.3 and 13.0, 3000 x 12288 72 and 83,
  // 12115 x 5544 90 and 96, 16384 x 4096 87 and 89; 8192 x 512 14.4 and 13.2, 4096 x 2048 21.5 and 18.5, 10000 x 768 20.5 and
  // 18.9.
  const int64_t most = n <= 2048 && blocks >= 2048 ? 512 : 256;
  return (int32_t)(blocks < most ? blocks : most);
}

size_t norm_grad_partial(int64_t m, int64_t n, int outputs) {
  const int32_t blocks = norm_grad_blocks(m, n);
  return blocks == 1 && n <= kMaxHeld ? 0 : (size_t)outputs * (size_t)blocks * (size_t)n * 4;
}

hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t stream) {
  const bool sums = a.dw || a.db;
  hipError_t e = hipSuccess;
  if (a.blocks > 0) {
    with_element(dtype, [&](auto t) {
      using T = decltype(t);
      if (a.n > kMaxHeld) {
        if (a.dx) {
          k_norm_grad_wide<T><<<wide_grid(a.m), dim3(1024), 0, stream>>>(a);
          if ((e = hipGetLastError()) != hipSuccess) return;
        }
        if (sums) k_norm_columns_wide<T><<<dim3((uint32_t)div_up(a.n, 2048), (uint32_t)a.blocks), dim3(256), 0, stream>>>(a);
        return;
      }
      with_shape(a.n, [&](auto s) {
        using S = decltype(s);
        k_norm_grad<T, S><<<dim3((uint32_t)a.blocks), dim3(S::kBlock), 0, stream>>>(a);
      });
    });
    if (e == hipSuccess) e = hipGetLastError();
  }
  if (e == hipSuccess && sums && (a.blocks != 1 || a.n > kMaxHeld)) {
    dim3 grid = wide_grid(div_up(a.n, kJoinColumns));
    grid.z = a.dw && a.db ? 2 : 1;
    k_norm_join<<<grid, dim3(kJoinColumns * kJoinRows), 0, stream>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace smat
