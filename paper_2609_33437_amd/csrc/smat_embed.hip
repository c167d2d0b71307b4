// Token embedding for gfx950: rows of a table by id, and the table's gradient by sorted tokens.
//
//   y_i = scale T[id_i],    dT[v] = scale sum over i with id_i = v of dy_i
//
// The gradient's tokens are sorted by id, those of one id staying in their order (a radix sort that counts, adds up and
// places one digit a pass).  A wave sums a chunk of sorted tokens, 64 eights of columns, and writes the rows whose tokens all
// lie in the chunk; the sums of runs that chunks cut go to the workspace and another launch adds them, in order.  No
// atomics, so a call's bits repeat.  Bound by HBM: dy is read once, and a gradient that is not accumulated writes every
// row of the table, zeros where no token is.
#include <type_traits>

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
// kLookups eights of columns a thread, their ids and then their rows loaded together.  An id outside the table gives a row of
// NaN.
constexpr int kLookups = 4;
template <typename T, typename U, typename Index>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a, Index across, int64_t total) {
  const int64_t first = wide_block() * (256 * kLookups) + threadIdx.x;
  Index row[kLookups];
  int64_t id[kLookups], j[kLookups];
  Raw8<T> raw[kLookups];
#pragma unroll
  for (int k = 0; k < kLookups; ++k) {
    const int64_t t = first + k * 256;
    row[k] = (Index)(t < total ? t : total - 1) / across;
    j[k] = (int64_t)((Index)(t < total ? t : total - 1) - row[k] * across) * 8;
    id[k] = a.ids[row[k]];
  }
#pragma unroll
  for (int k = 0; k < kLookups; ++k) {
    const bool in = id[k] >= 0 && id[k] < a.rows;
    raw[k].load_some(static_cast<const typename El<T>::Mem*>(a.table) + (in ? id[k] : 0) * a.ldt + j[k], in ? a.d - j[k] : 0);
  }
#pragma unroll
  for (int k = 0; k < kLookups; ++k) {
    if (first + k * 256 >= total) return;
    float v[8];
    raw[k].get(v);
    const bool in = id[k] >= 0 && id[k] < a.rows;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = in ? v[e] * a.scale : __builtin_nanf("");
    store_row8<U>(static_cast<typename El<U>::Mem*>(a.out) + (int64_t)row[k] * a.ldout + j[k], a.d - j[k], v);
  }
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

// ---------------------------------------------------------------- clearing
// A block of kSortThreads clears kClearEights eights a thread that follow each other over the block.  Rows end to end are
// one row, whose whole 16 bytes are written at their addresses.
constexpr int kClearEights = 8;
struct ClearArgs {
  void* table;
  int64_t ld, rows, d;
  int64_t before;  // elements up to the first 16-byte address of rows end to end
  int64_t eights;  // in all
};

template <typename U>
__device__ __forceinline__ void clear_block(const ClearArgs& c, int64_t block) {
  auto* out = static_cast<typename El<U>::Mem*>(c.table);
  const int64_t first = block * kSortThreads * kClearEights + threadIdx.x;
  const float v[8] = {};
  if (c.ld == c.d) {
    const int64_t n = c.rows * c.d - c.before;
    if (first < c.before) El<U>::store(out + first, 0.f);
#pragma unroll
    for (int k = 0; k < kClearEights; ++k) {
      const int64_t j = (first + k * kSortThreads) * 8;
      store_row8<U>(out + c.before + j, n - j, v);
    }
    return;
  }
  const int64_t across = (c.d + 7) / 8;
#pragma unroll 1
  for (int k = 0; k < kClearEights; ++k) {
    const int64_t t = first + k * kSortThreads;
    if (t >= c.eights) return;
    const int64_t row = c.eights <= INT64_C(0x7FFFFFFF) ? (int64_t)((uint32_t)t / (uint32_t)across) : t / across;
    const int64_t j = (t - row * across) * 8;
    store_row8<U>(out + row * c.ld + j, c.d - j, v);
  }
}

// ---------------------------------------------------------------- the sort of many tokens
// A pass counts a digit of each tile's tokens, adds the counts up, and places the tokens.  Blocks of the first pass's count clear
// the gradient meanwhile.
struct SortPass {
  const uint32_t* keys;    // NULL: the first pass, from the ids
  const uint32_t* places;
  uint32_t* keys_to;
  uint32_t* places_to;
  uint32_t* counts;        // [digits][tiles]
  int64_t tiles;
  int32_t shift, bits, summed;
};
constexpr int64_t kAddedTiles = 64;  // up to so many tiles' counts are added up by each placing block: a launch less a pass

template <typename U>
__global__ __launch_bounds__(kSortThreads) void k_sort_count(EmbedGradArgs a, SortPass s, ClearArgs c) {
  __shared__ uint32_t count[kMaxDigits];
  if (wide_block() >= s.tiles) {
    clear_block<U>(c, wide_block() - s.tiles);
    return;
  }
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

// counts <- their exclusive sums, by one block, where the tiles are too many for each block to add them up itself.
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
  __shared__ uint32_t waves[kSortWaves];
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
  // a digit's first place: after all lower digits, and the digit's in earlier tiles
  uint32_t place0 = 0, total;
  if (s.summed) {
    if (threadIdx.x < digits) place0 = s.counts[(int64_t)threadIdx.x * s.tiles + blockIdx.x];
    __syncthreads();
  } else {
    uint32_t all = 0;
    if (threadIdx.x < digits) {
      for (int64_t k = 0; k < s.tiles; ++k) {
        const uint32_t c = s.counts[(int64_t)threadIdx.x * s.tiles + k];
        place0 += k < blockIdx.x ? c : 0u;
        all += c;
      }
    }
    place0 += block_before(all, waves, &total);
  }
  if (threadIdx.x < digits) {
    uint32_t before = place0;
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

// ---------------------------------------------------------------- the sort of few tokens
// A gradient of no tokens.
template <typename U>
__global__ __launch_bounds__(kSortThreads) void k_embed_clear(ClearArgs c) {
  clear_block<U>(c, wide_block());
}

// Up to kOneSort tokens are sorted in LDS by the first block, a wave's tokens consecutive, with their digits' places
// counted as above.  The launch's other blocks clear the gradient meanwhile: 525 MB take 80 us, 6.6 TB/s, and the sort of
// 4096 tokens 15 us of them.
constexpr int64_t kOneSort = 16384;

struct OneSort {
  EmbedGradArgs a;
  ClearArgs clear;
  uint32_t* keys;
  uint32_t* places;
  int32_t bits, passes;
};

template <typename U, int ROUNDS>
__global__ __launch_bounds__(kSortThreads) void k_embed_order(OneSort o) {
  constexpr int kHeld = ROUNDS * kSortThreads;
  __shared__ uint32_t keys[kHeld];
  __shared__ uint16_t places[kHeld];
  __shared__ uint32_t count[kSortWaves][kMaxDigits];
  __shared__ uint32_t waves[kSortWaves];
  if (wide_block() != 0) {
    clear_block<U>(o.clear, wide_block() - 1);
    return;
  }
  const EmbedGradArgs& a = o.a;
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, first = wave * 64 * ROUNDS + lane, m = (int)a.m;
  uint32_t key[ROUNDS], at[ROUNDS];
  uint16_t place[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = first + r * 64;
    key[r] = i < m ? token_key(a, i) : 0u;
    place[r] = (uint16_t)i;
  }
  int32_t shift = 0, left = o.bits;
  for (int p = 0; p < o.passes; ++p) {
    const int bits = (left + o.passes - p - 1) / (o.passes - p);
    const uint32_t mask = (1u << bits) - 1u;
    for (int k = (int)threadIdx.x; k < kSortWaves * kMaxDigits; k += kSortThreads) (&count[0][0])[k] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) at[r] = wave_place((key[r] >> shift) & mask, bits, first + r * 64 < m, count[wave]);
    __syncthreads();
    // places of a digit's tokens of a wave: after all lower digits, and the digit's in earlier waves.  A thread adds up four
    // waves' of a digit.
    uint32_t c[4], total;
    const int digit = (int)threadIdx.x >> 2, w0 = ((int)threadIdx.x & 3) * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = count[w0 + k][digit];
    uint32_t before = block_before(c[0] + c[1] + c[2] + c[3], waves, &total);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      count[w0 + k][digit] = before;
      before += c[k];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (first + r * 64 < m) {
        const uint32_t to = count[wave][(key[r] >> shift) & mask] + at[r];
        keys[to] = key[r];
        places[to] = place[r];
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (first + r * 64 < m) {
        key[r] = keys[first + r * 64];
        place[r] = places[first + r * 64];
      }
    shift += bits;
    left -= bits;
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r)
    if (first + r * 64 < m) {
      o.keys[first + r * 64] = key[r];
      o.places[first + r * 64] = place[r];
    }
}

// ---------------------------------------------------------------- sums of rows
struct RowArgs {
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

// A lane holds one of the next 64 keys and places, so that a token's address waits for no load of its own.
template <typename T, typename U>
__global__ __launch_bounds__(256) void k_embed_sum(RowArgs r) {
  constexpr int kAhead = 8;
  const EmbedGradArgs& a = r.a;
  const int lane = (int)threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t t = wide_block() * 4 + wave;
  const int64_t c = t / r.tiles;
  if (c >= r.chunks) return;
  const int32_t eight = (int32_t)(t - c * r.tiles) * 64 + lane;
  const int64_t j = (int64_t)eight * 8;
  const bool on = eight < r.across;
  const int64_t valid = on ? a.d - j : 0;
  const int64_t begin = c * r.chunk, end = begin + r.chunk < a.m ? begin + r.chunk : a.m;
  const uint32_t none = (uint32_t)a.rows;
  const auto* dy = static_cast<const typename El<T>::Mem*>(a.dy) + j;
  float* partial = r.partial + (c * 2 * r.across + eight) * 8;
  // the key before the chunk and after it: no key is 2^32 - 1
  const uint32_t before = begin > 0 ? r.keys[begin - 1] : 0xFFFFFFFFu, after = end < a.m ? r.keys[end] : 0xFFFFFFFFu;
  uint32_t key = 0;
  bool cut = false;  // whether the run that is being summed began in an earlier chunk
  float sum[8] = {};
  for (int64_t p0 = begin; p0 < end; p0 += 64) {
    const int64_t mine = p0 + lane < end ? p0 + lane : end - 1;
    const uint32_t keys = r.keys[mine], places = r.places[mine];
    const int count = (int)(end - p0 < 64 ? end - p0 : 64);
    if (p0 == begin) {
      key = (uint32_t)__builtin_amdgcn_readlane((int)keys, 0);
      cut = key == before;
    }
    for (int q = 0; q < count; q += kAhead) {
      Raw8<T> raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = q + u < count ? q + u : count - 1;
        const uint32_t place = (uint32_t)__builtin_amdgcn_readlane((int)places, at);
        raw[u].load_some(dy + (int64_t)place * a.lddy, valid);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (q + u >= count) break;
        const uint32_t next = (uint32_t)__builtin_amdgcn_readlane((int)keys, q + u);
        if (next != key) {  // the run's end
          if (on) {
            if (cut)
              El<float>::store8(partial, sum);
            else
              write_row<U>(a, key, j, sum);
          }
          cut = false;
          key = next;
          if (key == none) return;  // the rest has no row
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        }
        float v[8];
        raw[u].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
      }
    }
  }
  if (key == none || !on) return;
  if (cut)
    El<float>::store8(partial, sum);
  else if (after == key)
    El<float>::store8(partial + (int64_t)r.across * 8, sum);
  else
    write_row<U>(a, key, j, sum);
}

// The run that begins in chunk c and goes on behind it: its sums in the chunks' order.
template <typename U>
__global__ __launch_bounds__(256) void k_embed_join(RowArgs r) {
  const EmbedGradArgs& a = r.a;
  const int64_t t = wide_block() * 4 + ((int)threadIdx.x >> 6);
  const int64_t c = t / r.tiles;
  if (c + 1 >= r.chunks) return;
  const int32_t eight = (int32_t)(t - c * r.tiles) * 64 + ((int)threadIdx.x & 63);
  const int64_t begin = c * r.chunk, end = begin + r.chunk;
  // the keys on both sides of the chunk's ends, loaded together
  const uint32_t key = r.keys[end - 1], after = r.keys[end], first = r.keys[begin], before = r.keys[begin > 0 ? begin - 1 : 0];
  if (key == (uint32_t)a.rows || after != key) return;
  if (begin > 0 && first == key && before == key) return;  // an earlier chunk's
  // the last chunk that holds a token of the run: the lanes look at 64 chunks at a time
  int64_t low = c + 1, high = r.chunks;
  for (int64_t each; low + 1 < high; high = low + each < high ? low + each : high) {
    each = (high - low + 63) / 64;
    const int64_t probe = low + ((int)threadIdx.x & 63) * each;
    low += (__popcll(__ballot(probe < high && r.keys[probe < high ? probe * r.chunk : 0] == key)) - 1) * each;
  }
  if (eight >= r.across) return;
  const int64_t step = (int64_t)r.across * 16;
  const float* p = r.partial + (c * 2 * r.across + eight) * 8;
  float sum[8];
  El<float>::load8(p + (int64_t)r.across * 8, sum);
  constexpr int kAhead = 8;
  for (int64_t k = 1; k <= low - c; k += kAhead) {
    Raw8<float> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) raw[u].load(p + (k + u <= low - c ? k + u : k) * step);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float v[8];
      raw[u].get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += k + u <= low - c ? v[e] : 0.f;
    }
  }
  write_row<U>(a, key, (int64_t)eight * 8, sum);
}

// ---------------------------------------------------------------- a handful of tokens
// Up to kFewTokens tokens need no sort and no second launch: a wave takes a token and 64 eights of columns, and where no
// earlier token has the id it sums that id's rows in order; other waves clear the rows of kClearRows that no token has.
// (9 tokens of 256 x 288: 4 us, and 12 us in the three launches of more tokens.)
constexpr int64_t kFewTokens = 256;
constexpr int kClearRows = 8;

template <typename T, typename U>
__global__ __launch_bounds__(256) void k_embed_few(EmbedGradArgs a, int32_t across, int32_t tiles, int64_t sums) {
  __shared__ uint32_t keys[kFewTokens];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int m = (int)a.m;
  if ((int)threadIdx.x < m) keys[threadIdx.x] = token_key(a, threadIdx.x);
  __syncthreads();
  if (wide_block() >= sums) {
    const int64_t first = ((wide_block() - sums) * 4 + wave) * kClearRows;
    uint32_t taken = 0;
    for (int p = 0; p < m; p += 64) {
      const int64_t row = p + lane < m ? (int64_t)keys[p + lane] - first : -1;
#pragma unroll
      for (int k = 0; k < kClearRows; ++k) taken |= __ballot(row == k) ? 1u << k : 0u;
    }
    const float v[8] = {};
    for (int k = 0; k < kClearRows && first + k < a.rows; ++k) {
      if (taken >> k & 1u) continue;
      auto* out = static_cast<typename El<U>::Mem*>(a.dtable) + (first + k) * a.ldt;
#pragma unroll 4
      for (int64_t j = lane * 8; j < a.d; j += 512) store_row8<U>(out + j, a.d - j, v);
    }
    return;
  }
  const int64_t t = wide_block() * 4 + wave;
  const int64_t token = t / tiles;
  if (token >= m) return;
  const int32_t eight = (int32_t)(t - token * tiles) * 64 + lane;
  const int64_t j = (int64_t)eight * 8, valid = eight < across ? a.d - j : 0;
  const uint32_t key = keys[token];
  if (key == (uint32_t)a.rows) return;
  const auto* dy = static_cast<const typename El<T>::Mem*>(a.dy) + j;
  float sum[8] = {};
  for (int p = 0; p < m; p += 64) {
    uint64_t same = __ballot(p + lane < m && keys[p + lane] == key);
    if (p + 64 <= token ? same != 0 : p <= token && (same & ((uint64_t(1) << (token - p)) - 1))) return;  // an earlier one's
    while (same) {
      constexpr int kAhead = 4;
      Raw8<T> raw[kAhead];
      int count = 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = same ? p + __ffsll((unsigned long long)same) - 1 : (int)token;
        count += same != 0;
        same &= same - 1;
        raw[u].load_some(dy + (int64_t)at * a.lddy, valid);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float v[8];
        raw[u].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += u < count ? v[e] : 0.f;
      }
    }
  }
  if (eight < across) write_row<U>(a, key, j, sum);
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
        k_embed<decltype(t), decltype(u), Index><<<wide_grid(div_up(total, 256 * kLookups)), dim3(256), 0, stream>>>(a, (Index)across, total);
      });
    });
  });
  return hipGetLastError();
}

EmbedGradPlan embed_grad_plan(const EmbedGradArgs& a) {
  EmbedGradPlan p{};
  if (a.m <= kFewTokens || a.d == 0 || a.rows == 0) return p;
  // few tokens a wave where they are few; with many, as many chunks as keep the join's sums short
  p.chunk = 8;
  while (p.chunk * 2048 < a.m) p.chunk *= 2;
  p.chunks = div_up(a.m, p.chunk);
  while ((a.rows >> p.bits) > 0) ++p.bits;
  p.passes = (p.bits + 7) / 8;
  p.tiles = a.m <= kOneSort ? 0 : div_up(a.m, kSortTile);
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
  char* ws = static_cast<char*>(workspace);
  const auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
  SortPass s{nullptr, nullptr, nullptr, nullptr, words(plan.counts), plan.tiles, 0, 0, plan.tiles > kAddedTiles};
  if (a.m > 0 && a.m <= kFewTokens) {
    const int64_t tiles = div_up(across, 64), sums = div_up(a.m * tiles, 4);
    const int64_t clears = a.accumulate ? 0 : div_up(a.rows, 4 * kClearRows);
    with_element(table_dtype, [&](auto u) {
      with_element(dtype, [&](auto t) {
        k_embed_few<decltype(t), decltype(u)><<<wide_grid(sums + clears), dim3(256), 0, stream>>>(a, (int32_t)across, (int32_t)tiles, sums);
      });
    });
    return hipGetLastError();
  }
  ClearArgs c{a.dtable, a.ldt, a.rows, a.d};
  if (!a.accumulate) {
    const int64_t n = a.rows * a.d, bytes = table_dtype == 1 ? 2 : 4;
    c.before = (int64_t)(-reinterpret_cast<uintptr_t>(a.dtable) & 15u) / bytes;
    if (c.before > n) c.before = n;
    c.eights = a.ldt == a.d ? div_up(n - c.before, 8) : a.rows * across;
  }
  const int64_t clears = a.accumulate ? 0 : c.eights > 0 ? div_up(c.eights, kSortThreads * kClearEights) : 1;
  const bool one = a.m > 0 && a.m <= kOneSort;
  if (one) {
    const OneSort o{a, c, words(plan.keys[0]), words(plan.places[0]), plan.bits, plan.passes};
    with_element(table_dtype, [&](auto u) {
      using U = decltype(u);
      const auto order = [&](auto rounds) {
        k_embed_order<U, rounds()><<<wide_grid(1 + clears), dim3(kSortThreads), 0, stream>>>(o);
      };
      if (a.m <= kSortThreads)
        order(std::integral_constant<int, 1>());
      else if (a.m <= 4 * kSortThreads)
        order(std::integral_constant<int, 4>());
      else if (a.m <= 8 * kSortThreads)
        order(std::integral_constant<int, 8>());
      else
        order(std::integral_constant<int, 16>());
    });
    s.keys = o.keys;
    s.places = o.places;
  } else if (a.m == 0 && clears > 0) {
    with_element(table_dtype, [&](auto u) {
      k_embed_clear<decltype(u)><<<wide_grid(clears), dim3(kSortThreads), 0, stream>>>(c);
    });
  }
  if ((e = hipGetLastError()) != hipSuccess || a.m == 0) return e;
  int32_t left = plan.bits;
  for (int p = 0; p < plan.passes && !one; ++p) {
    s.bits = (left + plan.passes - p - 1) / (plan.passes - p);
    s.keys_to = words(plan.keys[p % 2]);
    s.places_to = words(plan.places[p % 2]);
    const dim3 grid((uint32_t)plan.tiles), block(kSortThreads);
    with_element(table_dtype, [&](auto u) {
      k_sort_count<decltype(u)><<<wide_grid(plan.tiles + (p == 0 ? clears : 0)), block, 0, stream>>>(a, s, c);
    });
    if (s.summed) k_sort_sum<<<dim3(1), block, 0, stream>>>(s.counts, plan.tiles << s.bits);
    k_sort_place<<<grid, block, 0, stream>>>(a, s);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    s.shift += s.bits;
    left -= s.bits;
    s.keys = s.keys_to;
    s.places = s.places_to;
  }
  RowArgs r{a, s.keys, s.places, reinterpret_cast<float*>(ws + plan.partial), plan.chunk, plan.chunks, (int32_t)across,
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
