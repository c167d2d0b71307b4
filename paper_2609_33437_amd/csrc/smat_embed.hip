// Token embedding for gfx950: rows of a table by id, and the table's gradient by sorted tokens.
//
//   y_i = scale T[id_i],    dT[v] = scale sum over i with id_i = v of dy_i
//
// The gradient's tokens are sorted by id, those of one id staying in their order (a radix sort that counts, adds up and
// places one digit a pass).  A wave sums a chunk of sorted tokens, 64 eights of columns, and writes the rows whose tokens all
// lie in the chunk; the sums of runs that chunks cut go to the workspace and another launch adds them, in order.  No
// atomics, so a call's bits repeat.  Bound by HBM: dy is read once, and a gradient that is not accumulated writes every
// row of the table, zeros where no token is.
#include "smat_decoder.h"
#include "smat_linear_dev.h"

namespace smat {
namespace {

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
template <typename F>
void with_element(int dtype, F&& fn) {
  if (dtype == 1)
    fn(Bf16());
  else
    fn(float());
}

// ---------------------------------------------------------------- lookup
// Eight columns a thread.  An id outside the table gives a row of NaN.
template <typename T, typename U, typename Index>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a, Index across, int64_t total) {
  const int64_t t = wide_block() * 256 + threadIdx.x;
  if (t >= total) return;
  const Index row = (Index)t / across;
  const int64_t j = (int64_t)((Index)t - row * across) * 8, valid = a.d - j;
  const int64_t id = a.ids[row];
  float v[8];
  if (id >= 0 && id < a.rows) {
    load_row8<T>(static_cast<const typename El<T>::Mem*>(a.table) + id * a.ldt + j, valid, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= a.scale;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_nanf("");
  }
  store_row8<U>(static_cast<typename El<U>::Mem*>(a.out) + (int64_t)row * a.ldout + j, valid, v);
}

// ---------------------------------------------------------------- sort
// Keys are ids; tokens without a row (ids outside the table, the padding id) have the key `rows` and come last.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kTileRounds = 4;
constexpr int64_t kSortTile = kSortThreads * kTileRounds;  // tokens a block of the sort's launches takes
constexpr int kMaxDigits = 256;

__device__ __forceinline__ uint32_t token_key(const EmbedGradArgs& a, int64_t i) {
  const int64_t id = a.ids[i];
  return (uint32_t)(id < 0 || id >= a.rows || id == a.padding ? a.rows : id);
}

// This lane's place among the wave's tokens of its digit so far, which `count` [digits] of the wave counts.
__device__ __forceinline__ uint32_t wave_place(uint32_t digit, int bits, bool on, uint32_t* count) {
  const int lane = (int)threadIdx.x & 63;
  uint64_t same = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((digit >> b) & 1u);
    same &= (digit >> b) & 1u ? set : ~set;
  }
  const uint64_t below = same & ((uint64_t(1) << lane) - 1);
  uint32_t first = 0;
  if (on && below == 0) first = atomicAdd(&count[digit], (uint32_t)__popcll(same));
  first = (uint32_t)__shfl((int)first, on ? __ffsll((unsigned long long)same) - 1 : lane);
  return first + (uint32_t)__popcll(below);
}

// Exclusive sums over the block of one value a thread; *total: the sum of all.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* waves, uint32_t* total) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  uint32_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t other = (uint32_t)__shfl_up((int)sum, d);
    if (lane >= d) sum += other;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = sum;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < kSortWaves; ++k) {
    if (k < wave) before += waves[k];
    all += waves[k];
  }
  *total = all;
  return before + sum - v;
}

struct SortPass {
  const uint32_t* keys;    // NULL: the first pass, from the ids
  const uint32_t* places;
  uint32_t* keys_to;
  uint32_t* places_to;
  uint32_t* counts;        // [digits][tiles]
  int64_t tiles;
  int32_t shift, bits;
};

__global__ __launch_bounds__(kSortThreads) void k_sort_count(EmbedGradArgs a, SortPass s) {
  __shared__ uint32_t count[kMaxDigits];
  const uint32_t digits = 1u << s.bits;
  if (threadIdx.x < kMaxDigits) count[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int64_t i = (int64_t)blockIdx.x * kSortTile + r * kSortThreads + threadIdx.x;
    if (i < a.m) atomicAdd(&count[((s.keys ? s.keys[i] : token_key(a, i)) >> s.shift) & (digits - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < digits) s.counts[(int64_t)threadIdx.x * s.tiles + blockIdx.x] = count[threadIdx.x];
}

// counts <- their exclusive sums, by one block.
__global__ __launch_bounds__(kSortThreads) void k_sort_sum(uint32_t* counts, int64_t n) {
  __shared__ uint32_t waves[kSortWaves];
  uint32_t before = 0;
  for (int64_t i0 = 0; i0 < n; i0 += kSortThreads) {
    const int64_t i = i0 + threadIdx.x;
    uint32_t total;
    const uint32_t v = i < n ? counts[i] : 0u, at = block_before(v, waves, &total);
    if (i < n) counts[i] = before + at;
    before += total;
  }
}

// Wave w of a block takes its tokens [w 64 kTileRounds, ..): the order within a digit is the tokens'.
__global__ __launch_bounds__(kSortThreads) void k_sort_place(EmbedGradArgs a, SortPass s) {
  __shared__ uint32_t count[kSortWaves][kMaxDigits];
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  const uint32_t digits = 1u << s.bits;
  for (int k = (int)threadIdx.x; k < kSortWaves * kMaxDigits; k += kSortThreads) count[k / kMaxDigits][k % kMaxDigits] = 0;
  __syncthreads();
  uint32_t key[kTileRounds], place[kTileRounds], at[kTileRounds];
  const int64_t first = (int64_t)blockIdx.x * kSortTile + wave * 64 * kTileRounds + lane;
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int64_t i = first + r * 64;
    const bool on = i < a.m;
    key[r] = on ? (s.keys ? s.keys[i] : token_key(a, i)) : 0u;
    place[r] = on ? (s.keys ? s.places[i] : (uint32_t)i) : 0u;
    at[r] = wave_place((key[r] >> s.shift) & (digits - 1), s.bits, on, count[wave]);
  }
  __syncthreads();
  if (threadIdx.x < digits) {
    uint32_t before = s.counts[(int64_t)threadIdx.x * s.tiles + blockIdx.x];
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = count[w][threadIdx.x];
      count[w][threadIdx.x] = before;
      before += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    if (first + r * 64 < a.m) {
      const uint32_t to = count[wave][(key[r] >> s.shift) & (digits - 1)] + at[r];
      s.keys_to[to] = key[r];
      s.places_to[to] = place[r];
    }
  }
}

// ---------------------------------------------------------------- sums of rows
struct RunArgs {
  EmbedGradArgs a;
  const uint32_t* keys;    // sorted
  const uint32_t* places;
  float* partial;          // [chunks][first, last][8 across]: sums of runs that a chunk's ends cut
  int64_t chunk, chunks;
  int32_t across, tiles;   // eights a row, and tiles of 64 of them
};

template <typename U>
__device__ __forceinline__ void write_row(const EmbedGradArgs& a, int64_t row, int64_t j, float v[8]) {
  typename El<U>::Mem* out = static_cast<typename El<U>::Mem*>(a.dtable) + row * a.ldt + j;
  const int64_t valid = a.d - j;
  float old[8] = {};
  if (a.accumulate) load_row8<U>(out, valid, old);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(v[e], a.scale, old[e]);
  store_row8<U>(out, valid, v);
}

template <typename T, typename U>
__global__ __launch_bounds__(256) void k_embed_sum(RunArgs r) {
  constexpr int kAhead = 8;
  const EmbedGradArgs& a = r.a;
  const int64_t t = wide_block() * 4 + ((int)threadIdx.x >> 6);
  const int64_t c = t / r.tiles;
  if (c >= r.chunks) return;
  const int32_t eight = (int32_t)(t - c * r.tiles) * 64 + ((int)threadIdx.x & 63);
  const int64_t j = (int64_t)eight * 8, valid = a.d - j;
  const bool on = eight < r.across;
  const int64_t begin = c * r.chunk, end = begin + r.chunk < a.m ? begin + r.chunk : a.m;
  const uint32_t none = (uint32_t)a.rows;
  float* partial = r.partial + (c * 2 * r.across + eight) * 8;
  uint32_t key = r.keys[begin];
  // whether the run that is being summed began in an earlier chunk
  bool cut = begin > 0 && r.keys[begin - 1] == key;
  float sum[8] = {};
  for (int64_t p0 = begin; p0 < end && key != none; p0 += kAhead) {
    uint32_t keys[kAhead];
    float v[kAhead][8];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t p = p0 + u < end ? p0 + u : end - 1;
      keys[u] = r.keys[p];
      load_row8<T>(static_cast<const typename El<T>::Mem*>(a.dy) + (int64_t)r.places[p] * a.lddy + j, on ? valid : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (p0 + u >= end) break;
      if (keys[u] != key) {  // the run's end
        if (on) {
          if (cut)
            El<float>::store8(partial, sum);
          else
            write_row<U>(a, key, j, sum);
        }
        cut = false;
        key = keys[u];
        if (key == none) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[u][e];
    }
  }
  if (key == none || !on) return;
  if (cut)
    El<float>::store8(partial, sum);
  else if (end < a.m && r.keys[end] == key)
    El<float>::store8(partial + (int64_t)r.across * 8, sum);
  else
    write_row<U>(a, key, j, sum);
}

// The run that begins in chunk c and goes on behind it: its sums in the chunks' order.
template <typename U>
__global__ __launch_bounds__(256) void k_embed_join(RunArgs r) {
  const EmbedGradArgs& a = r.a;
  const int64_t t = wide_block() * 4 + ((int)threadIdx.x >> 6);
  const int64_t c = t / r.tiles;
  if (c + 1 >= r.chunks) return;
  const int32_t eight = (int32_t)(t - c * r.tiles) * 64 + ((int)threadIdx.x & 63);
  const int64_t begin = c * r.chunk, end = begin + r.chunk;
  const uint32_t key = r.keys[end - 1];
  if (key == (uint32_t)a.rows || r.keys[end] != key) return;
  if (begin > 0 && r.keys[begin] == key && r.keys[begin - 1] == key) return;  // an earlier chunk's
  // the last chunk that holds a token of the run
  int64_t low = c + 1, high = r.chunks - 1;
  while (low < high) {
    const int64_t middle = (low + high + 1) / 2;
    if (r.keys[middle * r.chunk] == key)
      low = middle;
    else
      high = middle - 1;
  }
  if (eight >= r.across) return;
  const int64_t step = (int64_t)r.across * 16;
  const float* p = r.partial + (c * 2 * r.across + eight) * 8;
  float sum[8];
  El<float>::load8(p + (int64_t)r.across * 8, sum);
#pragma unroll 4
  for (int64_t k = c + 1; k <= low; ++k) {
    float v[8];
    El<float>::load8(p + (k - c) * step, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += v[e];
  }
  write_row<U>(a, key, (int64_t)eight * 8, sum);
}

// Zeros in every row.
template <typename U, typename Index>
__global__ __launch_bounds__(256) void k_embed_clear(EmbedGradArgs a, Index across, int64_t total) {
  const int64_t t = wide_block() * 256 + threadIdx.x;
  if (t >= total) return;
  const Index row = (Index)t / across;
  const int64_t j = (int64_t)((Index)t - row * across) * 8;
  const float v[8] = {};
  store_row8<U>(static_cast<typename El<U>::Mem*>(a.dtable) + (int64_t)row * a.ldt + j, a.d - j, v);
}

template <typename F>
void with_index(int64_t total, F&& fn) {
  if (total <= INT64_C(0x7FFFFFFF))
    fn(uint32_t());
  else
    fn(int64_t());
}
}  // namespace

hipError_t launch_embed(const EmbedArgs& a, int table_dtype, int dtype, hipStream_t stream) {
  const int64_t across = div_up(a.d, 8), total = a.m * across;
  with_element(table_dtype, [&](auto t) {
    with_element(dtype, [&](auto u) {
      with_index(total, [&](auto index) {
        using Index = decltype(index);
        k_embed<decltype(t), decltype(u), Index><<<wide_grid(div_up(total, 256)), dim3(256), 0, stream>>>(a, (Index)across, total);
      });
    });
  });
  return hipGetLastError();
}

EmbedGradPlan embed_grad_plan(const EmbedGradArgs& a) {
  EmbedGradPlan p{};
  if (a.m == 0 || a.d == 0 || a.rows == 0) return p;
  // few tokens a wave where they are few; with many, as many chunks as keep the join's sums short
  p.chunk = 32;
  while (p.chunk * 1024 < a.m) p.chunk *= 2;
  p.chunks = div_up(a.m, p.chunk);
  while ((a.rows >> p.bits) > 0) ++p.bits;
  p.passes = (p.bits + 7) / 8;
  p.tiles = div_up(a.m, kSortTile);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 15) & ~(size_t)15;
    return here;
  };
  for (int k = 0; k < 2; ++k) {
    p.keys[k] = take((size_t)a.m * 4);
    p.places[k] = take((size_t)a.m * 4);
  }
  p.counts = take((size_t)p.tiles * kMaxDigits * 4);
  p.partial = take((size_t)p.chunks * 2 * (size_t)div_up(a.d, 8) * 32);
  p.workspace = at;
  return p;
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, int dtype, int table_dtype, const EmbedGradPlan& plan,
                             void* workspace, hipStream_t stream) {
  hipError_t e = hipSuccess;
  const int64_t across = div_up(a.d, 8);
  if (!a.accumulate) {
    const int64_t total = a.rows * across;
    with_element(table_dtype, [&](auto u) {
      with_index(total, [&](auto index) {
        using Index = decltype(index);
        k_embed_clear<decltype(u), Index><<<wide_grid(div_up(total, 256)), dim3(256), 0, stream>>>(a, (Index)across, total);
      });
    });
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.m == 0) return e;
  char* ws = static_cast<char*>(workspace);
  const auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
  SortPass s{nullptr, nullptr, nullptr, nullptr, words(plan.counts), plan.tiles, 0, 0};
  int32_t left = plan.bits;
  for (int p = 0; p < plan.passes; ++p) {
    s.bits = (left + plan.passes - p - 1) / (plan.passes - p);
    s.keys_to = words(plan.keys[p % 2]);
    s.places_to = words(plan.places[p % 2]);
    const dim3 grid((uint32_t)plan.tiles), block(kSortThreads);
    k_sort_count<<<grid, block, 0, stream>>>(a, s);
    k_sort_sum<<<dim3(1), block, 0, stream>>>(s.counts, plan.tiles << s.bits);
    k_sort_place<<<grid, block, 0, stream>>>(a, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    s.shift += s.bits;
    left -= s.bits;
    s.keys = s.keys_to;
    s.places = s.places_to;
  }
  RunArgs r{a, s.keys, s.places, reinterpret_cast<float*>(ws + plan.partial), plan.chunk, plan.chunks, (int32_t)across,
            (int32_t)div_up(across, 64)};
  const dim3 grid = wide_grid(div_up(r.chunks * r.tiles, 4));
  with_element(table_dtype, [&](auto u) {
    using U = decltype(u);
    with_element(dtype, [&](auto t) { k_embed_sum<decltype(t), U><<<grid, dim3(256), 0, stream>>>(r); });
    if (r.chunks > 1) k_embed_join<U><<<grid, dim3(256), 0, stream>>>(r);
  });
  return hipGetLastError();
}

}  // namespace smat
