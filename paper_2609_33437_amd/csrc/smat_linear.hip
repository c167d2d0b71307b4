// Linear-layer products for gfx950 on the matrix cores: the layer itself, its data gradient and its
// weight gradient, with their epilogues (see smat_linear.h for the operands).
//
// A block computes a tile of out.  Q's rows are the matrix instruction's rows and P's its columns, so a
// lane ends with consecutive j of one i; Q's rows are dealt to the instructions so that two of them
// leave a lane eight consecutive j (q_row), which is what the epilogues work on.
#include "smat_linear_dev.h"
#include "smat_launch.h"

namespace smat {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- operands in LDS
// A stage of an operand holds 128 bytes of r for each of its B rows or columns, in 16-byte chunks.
// Direct operands lie in rows of 8 chunks, transposed ones in rows of one r with B / (16 / bytes) chunks.
// A fragment is what a matrix step over 64 bytes of r reads: for bf16 lane l holds r = 8 (l / 16) .. + 8 of
// row l % 16 (one 32-deep instruction), for fp32 r = 4 (l / 16) .. + 4 (four 4-deep instructions, one
// element each).
//
// Chunks are exchanged within their row (an exclusive or) so that the lanes that read together reach
// different banks: by the row's number in P, and in Q, whose lanes read rows q_row, by the bits of the row
// that differ between them.  Direct operands have no conflicts so.  Transposed ones keep some: a quarter to a third of the
// active LDS cycles with 128 columns a stage, where the exchange has all its bits, and 0.61 of them with 64 (a weight gradient
// of 1999; 2048 x 257), whose rows have half as many chunks; with 32 Q's chunks are not exchanged at all.
__device__ __forceinline__ constexpr int q_row(int r, int t) { return (r >> 2) * 8 + t * 4 + (r & 3); }
template <bool Q>
__device__ __forceinline__ int direct_swizzle(int row) {
  return Q ? ((row & 3) | ((row >> 1) & 4)) : (row & 7);
}
// Transposed rows: lanes of one read lie in rows r = 8 g + (0..3), g < 4
// (bf16), or r = 4 g (fp32).
template <typename T, bool Q, int B>
__device__ __forceinline__ int transposed_swizzle(int r) {
  constexpr int kChunks = B * El<T>::kBytes / 16;
  if (El<T>::kBytes == 4) return (Q ? ((r >> 2) & 1) * 8 + ((r >> 3) & 1) : ((r >> 2) & 3) * 4) & (kChunks - 1);
  return (Q ? (r & 3) * 4 : ((r & 3) | ((r >> 1) & 4)) * 2) & (kChunks - 1);
}

// fn(0), fn(1), .., fn(N - 1) with constants.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void for_each(F&& fn) {
  if constexpr (I < N) {
    fn(std::integral_constant<int, I>());
    for_each<N, I + 1>(fn);
  }
}

template <typename T>
struct Frag;
template <>
struct Frag<Bf16> {
  bf16x8 v;
};
template <>
struct Frag<float> {
  f32x4 v;
};
// Instruction E of a fragment pair's kSteps.  One fp32 instruction after another on the same sum waits for it, so
// callers go through all sums before the next E.
template <typename T>
constexpr int kSteps = 1;
template <>
constexpr int kSteps<float> = 4;
template <int E>
__device__ __forceinline__ void mma(const Frag<Bf16>& q, const Frag<Bf16>& p, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q.v, p.v, c, 0, 0, 0);
}
template <int E>
__device__ __forceinline__ void mma(const Frag<float>& q, const Frag<float>& p, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(q.v[E], p.v[E], c, 0, 0, 0);
}

// The fragment of rows row0 .. row0 + 16 of P (of the pair's instruction t of rows row0 .. row0 + 32 of Q)
// over chunks 4 kk .. 4 kk + 4 of r, from a stage of B rows.
template <typename T, bool TRANS, bool Q, int B>
__device__ __forceinline__ Frag<T> read_frag(const char* stage, int row0, int t, int kk) {
  const int lane = (int)threadIdx.x & 63, g = lane >> 4, l = lane & 15;
  Frag<T> f;
  if constexpr (!TRANS) {
    const int row = row0 + (Q ? q_row(l, t) : l), c = (4 * kk + g) ^ direct_swizzle<Q>(row);
    f.v = *reinterpret_cast<const decltype(f.v)*>(stage + row * 128 + c * 16);
  } else if constexpr (sizeof(typename El<T>::Mem) == 2) {
    // each 16 lanes read four rows of r, 8 bytes a lane, and the instruction transposes them
    constexpr int kRow = B * 2;
    const int col = row0 + (Q ? (l & 3) * 8 + t * 4 : (l & 3) * 4);
    union {
      i16x4 h[2];
      bf16x8 v;
    } u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 32 * kk + 8 * g + 4 * h + (l >> 2);
      const int c = (col >> 3) ^ transposed_swizzle<T, Q, B>(r);
      const char* at = stage + r * kRow + c * 16 + (col & 4) * 2;
      u.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) i16x4*)const_cast<char*>(at));
    }
    f.v = u.v;
  } else {
    constexpr int kRow = B * 4;
    const int col = row0 + (Q ? q_row(l, t) : l);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * kk + 4 * g + e, c = (col >> 2) ^ transposed_swizzle<T, Q, B>(r);
      f.v[e] = *reinterpret_cast<const float*>(stage + r * kRow + c * 16 + (col & 3) * 4);
    }
  }
  return f;
}

// ---------------------------------------------------------------- operands of any alignment
// 16 bytes at any element's address where `valid` elements or more of them exist, else what there is, zeros after it.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const typename El<T>::Mem* p, int32_t valid) {
  constexpr int kChunk = 16 / El<T>::kBytes;
  typedef uint32_t word_mem __attribute__((aligned(2)));
  if (valid >= kChunk) return *reinterpret_cast<const typename El<T>::vec_mem*>(p);
  u32x4 x = {0u, 0u, 0u, 0u};
  if (valid <= 0) return x;
  const int32_t words = valid * El<T>::kBytes / 4;  // whole ones; bf16 may have half a word more
  const auto* w = reinterpret_cast<const word_mem*>(p);
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < words) x[e] = w[e];
  if constexpr (El<T>::kBytes == 2) {
    if (valid & 1) {
      const uint32_t half = p[valid - 1];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e == words) x[e] = half;
    }
  }
  return x;
}

// The epilogue of a wave's accumulators, or their store as a partial sum: four eights of values a lane at a
// time, chosen by a branch on a uniform number.  Unrolled over all 16 eights an epilogue with an activation is 100 KB
// of instructions that every tile reads anew; one eight at a time, its branches, its loads of other matrices and its
// stores wait for each other (12 us a tile of 256 x 256, against 6.5 us for four).  The next four's loads are asked for
// before these four's stores, which a wait for loads asked for later would include (a gated gradient of
// 4096 x 8960 x 1536 takes 179 us, 183 us with the loads after the stores).
// Instruction tile p of the accumulators lies ROWS(p) rows below i0, pair q COLS(q) columns right of j0.
template <typename T, int EPI, bool WHOLE, int NI, int NJ, typename R, typename C>
__device__ __forceinline__ void finish_eights(const LinArgs& a, int64_t i0, int64_t j0, const f32x4 (&acc)[NI][NJ],
                                              R rows, C cols) {
  constexpr int kEights = NI * NJ / 2, kAhead = WHOLE ? 4 : 1;
  const bool partial = a.splits > 1;
  const int64_t ld = (a.j + 7) & ~(int64_t)7;
  Side<T, EPI> side[kAhead];
  ColumnSide<T, EPI> column;
  const auto load = [&](int which, ColumnSide<T, EPI>& c, Side<T, EPI> (&s)[kAhead]) {
    const int64_t j = j0 + cols(which / NI);
    column_load<T, EPI>(a, j, c);
#pragma unroll
    for (int n = 0; n < kAhead; ++n) side_load<T, EPI, WHOLE>(a, i0 + rows(which % NI + n), j, s[n]);
  };
  if (!partial) load(0, column, side);
#pragma unroll 1
  for (int first = 0; first < kEights; first += kAhead) {
    const int which = __builtin_amdgcn_readfirstlane(first);
    float v[kAhead][8];
    Side<T, EPI> next_side[kAhead];
    ColumnSide<T, EPI> next_column;
    const int64_t j = j0 + cols(which / NI);
    if (!partial && which + kAhead < kEights) load(which + kAhead, next_column, next_side);
#pragma unroll
    for (int c = 0; c < kEights; c += kAhead) {
      if (which == c) {
        asm volatile("" ::: "memory");  // a branch, not a select for each value
#pragma unroll
        for (int n = 0; n < kAhead; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[n][e] = acc[(c + n) % NI][c / NI * 2][e];
            v[n][4 + e] = acc[(c + n) % NI][c / NI * 2 + 1][e];
          }
      }
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const int64_t i = i0 + rows(which % NI + n);
      if (partial) {
        if (WHOLE || (i < a.i && j < ld))
          El<float>::store8(a.partial + ((int64_t)blockIdx.y * a.i + i) * ld + j, v[n]);
      } else {
        epilogue8<T, EPI, 16, 32, WHOLE>(a, i, j, v[n], column, side[n]);
      }
    }
    column = next_column;
#pragma unroll
    for (int n = 0; n < kAhead; ++n) side[n] = next_side[n];
  }
}

// ROWS and COLS of the last tile and pair bound the wave's part of the tile.
template <typename T, int EPI, int NI, int NJ, typename R, typename C>
__device__ __forceinline__ void finish(const LinArgs& a, int64_t i0, int64_t j0, const f32x4 (&acc)[NI][NJ], R rows,
                                       C cols) {
  static_assert(NI % 4 == 0, "four eights of one pair at a time");
  const int lane = (int)threadIdx.x & 63, g = lane >> 4, l = lane & 15;
  if (i0 + rows(NI - 1) + 16 <= a.i && j0 + cols(NJ / 2 - 1) + 32 <= a.j)
    finish_eights<T, EPI, true>(a, i0 + l, j0 + 8 * g, acc, rows, cols);
  else
    finish_eights<T, EPI, false>(a, i0 + l, j0 + 8 * g, acc, rows, cols);
}

// The first of range s's stages where n < 2^27 stages are dealt to `splits` ranges.
__device__ __forceinline__ int64_t split_start(int64_t n, uint32_t s, int32_t splits) {
  const uint32_t each = (uint32_t)n / (uint32_t)splits, more = (uint32_t)n - each * (uint32_t)splits;
  return (int64_t)(each * s + (s < more ? s : more));
}

// ---------------------------------------------------------------- the pipelined tile
// bf16 operands whose rows start on 16-byte boundaries (and, where r runs along them, end on one) go
// from global memory to LDS without passing registers.
//
// A tile of 256 x 256 is computed by eight waves; a stage (64 r) of each operand lies in LDS in two halves of
// 128 rows or columns, twice, 128 KB in all.  A wave computes 64 x 32 of each of the four quadrants in two phases
// a stage: the first reads P's first half and both halves of Q (16 fragments) and multiplies them, the second
// reads P's second half.  Between its reads and its 32 matrix instructions a phase starts the copies
// into the halves that the previous phase emptied.  Waves 4 to 7 run half a phase behind waves 0 to 3, so on
// each SIMD one wave's matrix instructions cover the other's memory instructions.  (With one quadrant a phase the
// barriers left the matrix cores idle for a quarter of the time.)
//
// Bound by the matrix cores: 8192 x 4096 x 14336 with a residual takes 670 us, 1430 TFLOP/s, with them busy 90 % of the
// time; a weight gradient of the same size, both operands transposed, 1370 TFLOP/s and 82 %.  256 x 256 is the largest
// tile whose sums (128 registers a lane) and whose two stages (128 KB) a compute unit holds, and so reads LDS least.
//
// What orders the phases: a wave passes the barrier before its matrix instructions once its own reads of LDS have
// returned and all but its last 8 copies (four halves) have landed.  So a half is read after a barrier
// that every wave passed with its share of it landed, and a copy into a half starts after a barrier that every wave
// passed with its reads of it returned.  Copies past the last stage deliver zeros to places that
// nothing reads; they keep the count.
constexpr int kFastB = 256, kFastThreads = 512, kFastHalf = 128, kHalfBytes = kFastHalf * 128;

typedef __attribute__((address_space(3))) char lds_char;
typedef int i32x4 __attribute__((ext_vector_type(4)));

// A buffer descriptor of `bytes` bytes: offsets past them read as zeros.
__device__ __forceinline__ i32x4 make_rsrc(uint64_t p, uint32_t bytes) {
  return i32x4{(int)(uint32_t)p, (int)((uint32_t)(p >> 32) & 0xFFFFu), (int)bytes, 0x00020000};
}
// 16 bytes a lane from `offset` of the buffer to LDS bytes lds + PLUS + 16 lane.
template <int PLUS>
__device__ __forceinline__ void copy_to_lds(i32x4 rsrc, uint32_t offset, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(offset), "s"(rsrc), "n"(PLUS)
               : "memory", "scc");
}
constexpr uint32_t kNowhere = 0x80000000u;  // past the end of every buffer

constexpr uint32_t kMaxCopies = 63;  // what a wait can leave in flight

// The wave's own reads of LDS have returned.  A builtin, so that the compiler knows; it would wait again later, for
// reads that were asked for in between too.
__device__ __forceinline__ void wait_reads() {
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0), any vmcnt and expcnt
  asm volatile("" ::: "memory");
}
// All but N of its copies have landed, and its reads have returned.
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N <= (int)kMaxCopies, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
  wait_reads();
}

// Where the next stage of an operand lies, as the copies take it.
template <typename T, bool TRANS, bool Q>
struct Stream {
  static constexpr int kBytes = El<T>::kBytes, kDeep = 128 / kBytes;
  uint64_t base, step;
  uint32_t bytes;  // offsets past them read as zeros
  // rows (columns) from row0 on, stage number `at` of the product
  __device__ __forceinline__ void set(const LinProduct& pr, int64_t row0, int64_t at) {
    const int64_t ld = Q ? pr.ldq : pr.ldp, r0 = at * kDeep;
    base = reinterpret_cast<uint64_t>(Q ? pr.q : pr.p) + (uint64_t)(TRANS ? r0 * ld + row0 : row0 * ld + r0) * kBytes;
    step = TRANS ? (uint64_t)ld * 128 : 128;
    bytes = 0x7FFFFFF0u;
  }
  // the stage has `deep` r and is the product's last: a transposed one ends with its last row's last column, to whole 16
  __device__ __forceinline__ void end(const LinProduct& pr, int64_t row0, int64_t rows, int32_t deep) {
    if constexpr (TRANS) {
      const int64_t some = row0 < rows ? (((deep - 1) * (Q ? pr.ldq : pr.ldp) + rows - row0) * kBytes + 15) & ~(int64_t)15 : 0;
      bytes = (uint32_t)(some < 0x7FFFFFF0 ? some : 0x7FFFFFF0);
    }
  }
  __device__ __forceinline__ i32x4 rsrc() const { return make_rsrc(base, bytes); }
};

// The stages of r that a block (a group) takes, in the order of the sum: those of prod[0], then those of prod[1].  Runs of
// whole stages are passed by additions alone, since what a stage adds to a wave's instructions delays its matrix
// instructions; a product's last stage and the end of the share are set up apart.
// set(product) deals the operands' rows to the copies, end(r) cuts the copies of direct operands to the first r of the stage.
template <typename T, bool PT, bool QT>
struct Feed {
  static constexpr int kDeep = 128 / El<T>::kBytes;
  Stream<T, PT, false> p;
  Stream<T, QT, true> q;
  int64_t i0, j0;
  int32_t plain;              // stages left of this run
  int32_t run, at, last, second;  // its length, its first stage and the share's end in its product, whether that is prod[1]
  int32_t last_second;        // the share's end in prod[1]

  template <typename Set, typename End>
  __device__ __forceinline__ void begin(const LinArgs& a, int64_t i0_, int64_t j0_, int64_t first, int64_t end_, int64_t n0,
                                        Set set, End end) {
    i0 = i0_;
    j0 = j0_;
    second = first >= n0 && a.prod[1].r > 0;
    at = (int32_t)(second ? first - n0 : first);
    last_second = (int32_t)(end_ - n0);
    last = second ? last_second : (int32_t)(end_ < n0 ? end_ : n0);
    set(a.prod[second]);
    next_run(a, n0, set, end);
  }
  template <typename Set, typename End>
  __device__ __forceinline__ void next_run(const LinArgs& a, int64_t n0, Set set, End end) {
    if (at >= last && !second && last_second > 0) {
      second = 1;
      at = 0;
      last = last_second;
      set(a.prod[1]);
    }
    const LinProduct& pr = a.prod[second];
    p.set(pr, i0, at);
    q.set(pr, j0, at);
    if (at >= last) {  // none is left: what is copied from here on are zeros
      p.bytes = q.bytes = 0;
      p.step = q.step = 0;
      end(0);
      run = INT32_MAX;
    } else {
      const int32_t whole = (int32_t)((pr.r + kDeep - 1) / kDeep) - 1;  // the product's last stage
      run = (whole < last ? whole : last) - at;
      if (run <= 0) {
        const int32_t deep = (int32_t)(pr.r - (int64_t)at * kDeep);
        p.end(pr, i0, a.i, deep);
        q.end(pr, j0, a.j, deep);
        end(deep);
        run = 1;
      }
    }
    plain = run;
  }
  template <typename Set, typename End>
  __device__ __forceinline__ void advance(const LinArgs& a, int64_t n0, Set set, End end) {
    p.base += p.step;
    q.base += q.step;
    if (--plain == 0) {
      at += run;
      next_run(a, n0, set, end);
    }
  }
};

// Copies of NI KB of a stage by one of the waves that share it: B rows (columns), the first `skip` behind the stream's.
template <typename T, bool TRANS, bool Q, int B, int NI>
struct Copy {
  static constexpr int kBytes = El<T>::kBytes, kChunk = 16 / kBytes;
  uint32_t off[NI];  // this lane's bytes from the stream's place
  static __device__ __forceinline__ int chunk_of(int u, int wave, int& row) {
    const int lane = (int)threadIdx.x & 63;
    row = (wave * NI + u) * 8 + lane / 8;
    return (lane % 8) ^ direct_swizzle<Q>(row);
  }
  // rows: the operand's from the stream's first on
  __device__ __forceinline__ void set(const LinProduct& pr, int skip, int64_t rows, int wave) {
    const int lane = (int)threadIdx.x & 63;
    const uint32_t ld = (uint32_t)(Q ? pr.ldq : pr.ldp);
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      if constexpr (!TRANS) {
        int row;
        const int c = chunk_of(u, wave, row);
        off[u] = skip + row < rows ? (uint32_t)(skip + row) * ld * kBytes + (uint32_t)c * 16 : kNowhere;
      } else {
        constexpr int kChunks = B / kChunk;
        const int rr = (wave * NI + u) * (64 / kChunks) + lane / kChunks;
        const int c = (lane % kChunks) ^ transposed_swizzle<T, Q, B>(rr);
        // chunks lie inside their row's stride (a multiple of 16 bytes) as long as their first column does
        off[u] = skip + c * kChunk < rows ? (uint32_t)rr * ld * kBytes + (uint32_t)(skip * kBytes + c * 16) : kNowhere;
      }
    }
  }
  // The stage has only `left` r: the chunks past them lie nowhere, here and until set().
  __device__ __forceinline__ void end(int32_t left, int wave) {
    if constexpr (!TRANS) {
#pragma unroll
      for (int u = 0; u < NI; ++u) {
        int row;
        if (chunk_of(u, wave, row) * kChunk >= left) off[u] = kNowhere;
      }
    }
  }
  // KB U of the stage at rsrc into LDS bytes `lds` .. of this wave's first KB
  template <int U>
  __device__ __forceinline__ void one(i32x4 rsrc, uint32_t lds) const {
    copy_to_lds<U * 1024>(rsrc, off[U], lds);
  }
  template <int U = 0>
  __device__ __forceinline__ void all(i32x4 rsrc, uint32_t lds) const {
    if constexpr (U < NI) {
      one<U>(rsrc, lds);
      all<U + 1>(rsrc, lds);
    }
  }
};

// The same stages by way of registers, for operands of any alignment and stride.
template <typename T, bool TRANS, bool Q, int B, int NI>
struct Staged {
  static constexpr int kBytes = El<T>::kBytes, kChunk = 16 / kBytes, kDeep = 128 / kBytes;
  static constexpr int kAcross = TRANS ? B / kChunk : 8;  // chunks a row of the stage
  static constexpr int kRows = 64 / kAcross;              // rows of the stage a KB
  const typename El<T>::Mem* base;                        // of the first row or column
  int64_t ld, r, r0;  // r0: of the next stage
  int32_t left;       // rows or columns from the first one, as far as the stage reaches
  int32_t row, c;     // this lane's row of the stage in the first KB, and its chunk
  int64_t off;        // its elements from base at r0 = 0
  u32x4 x[NI];
  __device__ __forceinline__ void set(const LinProduct& pr, int64_t row0, int64_t rows, int64_t from, int wave) {
    const int lane = (int)threadIdx.x & 63;
    r = pr.r;
    r0 = from;
    ld = Q ? pr.ldq : pr.ldp;
    left = (int32_t)(rows - row0 < B ? rows - row0 : B);
    base = static_cast<const typename El<T>::Mem*>(Q ? pr.q : pr.p) + (TRANS ? row0 : row0 * ld);
    row = wave * NI * kRows + lane / kAcross;
    c = lane % kAcross;
    off = row * ld + c * kChunk;
  }
  __device__ __forceinline__ void load(bool on) {
    // r of this stage, <= 0 past the last
    const int32_t deep = on ? (int32_t)(r - r0 < kDeep ? r - r0 : kDeep) : 0;
    const int32_t short_ld = (int32_t)(ld < kChunk ? ld : kChunk);
    const auto* p = base + (TRANS ? r0 * ld : r0);
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int32_t at = row + u * kRows;
      int32_t valid;
      if constexpr (TRANS)
        // a chunk may run past its row into the next ones, whose values only reach columns outside, but not
        // past the last row of the stage
        valid = at < deep && c * kChunk < left ? (deep - 1 - at) * short_ld + left - c * kChunk : 0;
      else
        valid = at < left ? deep - c * kChunk : 0;
      x[u] = load_chunk<T>(p + u * kRows * ld + off, valid);
    }
  }
  __device__ __forceinline__ void next() { r0 += kDeep; }
  __device__ __forceinline__ void store(char* stage) const {
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int at = row + u * kRows;
      const int swizzled = TRANS ? c ^ transposed_swizzle<T, Q, B>(at) : c ^ direct_swizzle<Q>(at);
      *reinterpret_cast<u32x4*>(stage + at * (kAcross * 16) + swizzled * 16) = x[u];
    }
  }
};

// Tile `b` of ti x tj in an order that keeps the tiles that run together close: consecutive blocks go to the
// eight XCDs in turn, so each XCD takes one run of the order, in columns four tiles high.
__device__ __forceinline__ void tile_place(uint32_t b, uint32_t ti, uint32_t tj, uint32_t& i, uint32_t& j) {
  const uint32_t n = ti * tj, x = b & 7u, q = n >> 3, rem = n & 7u;
  const uint32_t t = x * q + (x < rem ? x : rem) + (b >> 3);
  constexpr uint32_t kHigh = 4;
  const uint32_t band = t / (kHigh * tj), in = t - band * kHigh * tj, high = ti - band * kHigh < kHigh ? ti - band * kHigh : kHigh;
  j = in / high;
  i = band * kHigh + (in - j * high);
}

template <bool PT, bool QT, int EPI>
__global__ __launch_bounds__(kFastThreads, 2) void k_linear_fast(LinArgs a) {
  using T = Bf16;
  extern __shared__ char smem[];  // [stage parity][P half 0, P half 1, Q half 0, Q half 1]
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
  uint32_t ti, tj;
  tile_place(blockIdx.x, (uint32_t)((a.i + kFastB - 1) / kFastB), (uint32_t)((a.j + kFastB - 1) / kFastB), ti, tj);
  const int64_t i0 = (int64_t)ti * kFastB, j0 = (int64_t)tj * kFastB;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wi = wave / 4 * 64, wj = wave % 4 * 32;
  const int64_t n0 = (a.prod[0].r + 63) / 64, n = n0 + (a.prod[1].r + 63) / 64;
  const int64_t first = split_start(n, blockIdx.y, a.splits), last = split_start(n, blockIdx.y + 1, a.splits);
  Feed<T, PT, QT> feed;
  Copy<T, PT, false, kFastHalf, 2> cp[2];
  Copy<T, QT, true, kFastHalf, 2> cq[2];
  const auto set = [&](const LinProduct& pr) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      cp[h].set(pr, h * kFastHalf, a.i - i0, wave);
      cq[h].set(pr, h * kFastHalf, a.j - j0, wave);
    }
  };
  const auto end = [&](int32_t deep) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      cp[h].end(deep, wave);
      cq[h].end(deep, wave);
    }
  };
  feed.begin(a, i0, j0, first, last, n0, set, end);
  const uint32_t mine = lds0 + (uint32_t)wave * 2048;
  const auto copy_p = [&](int h, int buf) {  // half h of the next stage to copy
    cp[h].all(feed.p.rsrc(), mine + (buf * 4 + h) * kHalfBytes);
  };
  const auto copy_q = [&](int h, int buf) { cq[h].all(feed.q.rsrc(), mine + (buf * 4 + 2 + h) * kHalfBytes); };
  const auto advance = [&] { feed.advance(a, n0, set, end); };
  f32x4 acc[8][4] = {};  // [half of P, tile][half of Q, tile]
  Frag<T> fp[4][2], fq[2][2][2];  // [tile][kk], [half][tile][kk]
  const auto read_p = [&](int h, int buf) {
    const char* s = smem + buf * 4 * kHalfBytes + h * kHalfBytes;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) fp[x][kk] = read_frag<T, PT, false, kFastHalf>(s, wi + 16 * x, 0, kk);
  };
  const auto read_q = [&](int h, int buf) {
    const char* s = smem + buf * 4 * kHalfBytes + (2 + h) * kHalfBytes;
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) fq[h][y][kk] = read_frag<T, QT, true, kFastHalf>(s, wj, y, kk);
  };
  const auto multiply = [&](int hp) {
    wait_copies<8>();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) mma<0>(fq[y / 2][y % 2][kk], fp[x][kk], acc[4 * hp + x][y]);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };
  // The stage in buffer `buf`.  The copies run ahead of it: P's second half by one stage, the others by two.
  const auto stage = [&](int buf) {
    read_p(0, buf);
    read_q(0, buf);
    read_q(1, buf);
    copy_p(1, buf ^ 1);
    advance();
    multiply(0);
    read_p(1, buf);
    copy_q(0, buf);
    copy_q(1, buf);
    copy_p(0, buf);
    multiply(1);
  };
  copy_q(0, 0);
  copy_q(1, 0);
  copy_p(0, 0);
  copy_p(1, 0);
  advance();
  copy_q(0, 1);
  copy_q(1, 1);
  copy_p(0, 1);
  asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if (wave >= 4) __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  for (int32_t s = (int32_t)(last - first); s > 0; s -= 2) {
    stage(0);
    if (s > 1) stage(1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no copy outlives the block's LDS
  if (wave < 4) __builtin_amdgcn_s_barrier();
  finish<T, EPI>(
      a, i0 + wi, j0 + wj, acc, [](int p) { return p / 4 * kFastHalf + p % 4 * 16; },
      [](int q) { return q * kFastHalf; });
}

// ---------------------------------------------------------------- smaller tiles
// The same copies and fragments for products that would leave the 256 x 256 tile's compute units idle.  A block holds
// G groups of WI x WJ waves.  A group computes the whole tile, TI x TJ a wave, over its own share of the
// stages of r; where G > 1 the groups' sums are added through LDS.  So a product with few tiles and a long r
// still keeps several waves' copies in flight on each compute unit, and no launch joins them.
//
// A group's stages lie in NBUF buffers.  While a wave multiplies the fragments of one stage it reads those of the
// next from LDS; a buffer is filled again once every wave of the group has read it.
//
// Where tiles are few these kernels are bound by what a block's waves can issue and by their start and end (128 x 128 with
// two groups: 0.95 us a step of two stages, 0.44 us of it in matrix instructions): 4096 x 1024 x 4096 takes 38.5 us,
// 890 TFLOP/s (47 us without the second group), 2048 x 2048 x 2048 23 us, 300 x 1024 x 1024 6.5 us.  In fp32 128 x 128
// tiles, two blocks a unit, are bound by the matrix cores: 4096 x 4096 x 4096 950 us, 145 TFLOP/s.
template <int TI_, int TJ_, int WI_, int WJ_, int G_, int NBUF_>
struct GroupShape {
  static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, G = G_, NBUF = NBUF_;
  using Staged = GroupShape<TI_, TJ_, WI_, WJ_, G_, 2>;      // as stages by way of registers need it
  static constexpr int kI = TI * WI, kJ = TJ * WJ, kThreads = 64 * WI * WJ * G;
  static constexpr int kStage = (kI + kJ) * 128;             // bytes
  static constexpr int kSumLd = kJ + 4;                      // floats a row of a group's sums (rows 16 bytes apart in banks)
  static constexpr int kSums = G > 1 ? G * kI * kSumLd * 4 : 0;
  static constexpr int kLds = G * NBUF * kStage > kSums ? G * NBUF * kStage : kSums;
  static constexpr int kResident = 160 * 1024 / kLds;        // blocks that fit a compute unit's LDS
  static constexpr int kSimdWaves = kResident * WI * WJ * G / 4;
};

// DIRECT: stages go from global memory to LDS (Copy), else through registers (Staged; two buffers).
template <typename T, bool PT, bool QT, int EPI, typename S, bool DIRECT>
__global__ __launch_bounds__(S::kThreads, S::kSimdWaves) void k_linear_group(LinArgs a) {
  constexpr int kWaves = S::WI * S::WJ, kNp = S::kI / 8 / kWaves, kNq = S::kJ / 8 / kWaves, kXi = S::TI / 16, kXj = S::TJ / 16;
  constexpr int kDeep = 128 / El<T>::kBytes;
  static_assert(kNp * 8 * kWaves == S::kI && kNq * 8 * kWaves == S::kJ, "whole KB a wave");
  static_assert(S::NBUF == 2 || DIRECT, "a stage in registers, one being read, one being written");
  extern __shared__ char smem[];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), group = wave / kWaves, w = wave % kWaves;
  uint32_t ti, tj;
  tile_place(blockIdx.x, (uint32_t)((a.i + S::kI - 1) / S::kI), (uint32_t)((a.j + S::kJ - 1) / S::kJ), ti, tj);
  const int64_t i0 = (int64_t)ti * S::kI, j0 = (int64_t)tj * S::kJ;
  const int wi = w / S::WJ * S::TI, wj = w % S::WJ * S::TJ;
  const int64_t n0 = (a.prod[0].r + kDeep - 1) / kDeep, n = n0 + (a.prod[1].r + kDeep - 1) / kDeep;
  const uint32_t share = blockIdx.y * S::G + (uint32_t)group;
  const int64_t first = split_start(n, share, a.splits * S::G), last = split_start(n, share + 1, a.splits * S::G);
  // every group of a block takes the same number of steps, so that barriers meet (shares differ by one stage)
  const int64_t steps = (n + a.splits * S::G - 1) / (a.splits * S::G);
  Feed<T, PT, QT> feed;
  Copy<T, PT, false, S::kI, kNp> cp;
  Copy<T, QT, true, S::kJ, kNq> cq;
  Staged<T, PT, false, S::kI, kNp> rp;
  Staged<T, QT, true, S::kJ, kNq> rq;
  const auto set = [&](const LinProduct& pr) {
    cp.set(pr, 0, a.i - i0, w);
    cq.set(pr, 0, a.j - j0, w);
  };
  const auto end = [&](int32_t deep) {
    cp.end(deep, w);
    cq.end(deep, w);
  };
  // by way of registers: the next stage's number, and of its product
  int64_t at = first;
  const auto stage_of = [&] {
    const bool second = at >= n0 && a.prod[1].r > 0;
    rp.set(a.prod[second], i0, a.i, (second ? at - n0 : at) * kDeep, w);
    rq.set(a.prod[second], j0, a.j, (second ? at - n0 : at) * kDeep, w);
  };
  if constexpr (DIRECT)
    feed.begin(a, i0, j0, first, last, n0, set, end);
  else
    stage_of();
  char* const mine = smem + group * S::NBUF * S::kStage;
  const uint32_t mine_p = (uint32_t)(uintptr_t)(lds_char*)mine + (uint32_t)(w * kNp * 1024);
  const uint32_t mine_q = (uint32_t)(uintptr_t)(lds_char*)mine + (uint32_t)(S::kI * 128 + w * kNq * 1024);
  const auto advance = [&] {
    if constexpr (DIRECT) {
      feed.advance(a, n0, set, end);
    } else {
      rp.next();
      rq.next();
      if (++at == n0) stage_of();
    }
  };
  // the next stage on its way: into buffer `buf`, or into registers
  const auto fetch = [&](int buf) {
    if constexpr (DIRECT) {
      cp.all(feed.p.rsrc(), mine_p + (uint32_t)(buf * S::kStage));
      cq.all(feed.q.rsrc(), mine_q + (uint32_t)(buf * S::kStage));
    } else {
      rp.load(at < last);
      rq.load(at < last);
    }
    advance();
  };
  const auto place = [&](int buf) {
    if constexpr (!DIRECT) {
      rp.store(mine + buf * S::kStage);
      rq.store(mine + buf * S::kStage + S::kI * 128);
    }
  };
  f32x4 acc[kXi][kXj] = {};
  Frag<T> fp[2][kXi][2], fq[2][kXj][2];  // [parity][tile][kk]
  // fragment number n of a stage: P's and Q's of kk = 0, then of kk = 1
  constexpr int kFrags = 2 * (kXi + kXj);
  const auto read_one = [&](int set_, int buf, int n) {
    const char* s = mine + buf * S::kStage;
    const int kk = n / (kXi + kXj), x = n % (kXi + kXj), y = x - kXi;
    if (x < kXi)
      fp[set_][x][kk] = read_frag<T, PT, false, S::kI>(s, wi + 16 * x, 0, kk);
    else
      fq[set_][y][kk] = read_frag<T, QT, true, S::kJ>(s + S::kI * 128, wj + 32 * (y / 2), y % 2, kk);
  };
  const auto meet = [&] {
    if (kWaves > 1) {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("" ::: "memory");
    }
  };
  // a stage's products in kPieces parts: all Q of one row of P's tiles at one kk
  constexpr int kPieces = 2 * kXi;
  const auto multiply = [&](int set_, int piece) {
    const int kk = piece / kXi, x = piece % kXi;
    const auto all = [&](auto e) {
#pragma unroll
      for (int y = 0; y < kXj; ++y) mma<decltype(e)::value>(fq[set_][y][kk], fp[set_][x][kk], acc[x][y]);
    };
    all(std::integral_constant<int, 0>());
    if constexpr (kSteps<T> == 4) {
      all(std::integral_constant<int, 1>());
      all(std::integral_constant<int, 2>());
      all(std::integral_constant<int, 3>());
    }
  };
  int buf = 0;
  // The fragments `set_` of this step have been asked for.  DIRECT: wait for them and for the next stage, then fill their
  // buffer again, ask for the next fragments and multiply.  Else: put the next stage into the other buffer (whose
  // fragments every wave had before the last barrier), start loading the one after, wait, and the same.  The copies and
  // reads are dealt out between the matrix instructions, which run on while a wave issues them: fp32
  // 2056 x 4096 x 1024 takes 138 us so, and 146 us with all of them first.
  const auto step = [&](int set_) {
    i32x4 rsrc_p, rsrc_q;
    uint32_t to_p = 0, to_q = 0;
    if constexpr (DIRECT) {
      rsrc_p = feed.p.rsrc();
      rsrc_q = feed.q.rsrc();
      to_p = mine_p + (uint32_t)(buf * S::kStage);
      to_q = mine_q + (uint32_t)(buf * S::kStage);
      wait_copies<(S::NBUF - 2) * (kNp + kNq)>();
      meet();
      buf = buf + 1 == S::NBUF ? 0 : buf + 1;
    } else {
      buf ^= 1;
      place(buf);
      fetch(buf);
      wait_reads();
      meet();
    }
    for_each<kPieces>([&](auto piece) {
      constexpr int kFirst = piece * (kNp + kNq) / kPieces, kEnd = (piece + 1) * (kNp + kNq) / kPieces;
      multiply(set_, piece);
      if constexpr (DIRECT) {
        for_each<kEnd - kFirst>([&](auto d) {
          constexpr int u = kFirst + d;
          if constexpr (u < kNp)
            cp.template one<u>(rsrc_p, to_p);
          else
            cq.template one<u - kNp>(rsrc_q, to_q);
        });
      }
#pragma unroll
      for (int n = piece * kFrags / kPieces; n < (piece + 1) * kFrags / kPieces; ++n) read_one(set_ ^ 1, buf, n);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (DIRECT) advance();
  };
  if constexpr (DIRECT) {
#pragma unroll
    for (int b = 0; b < S::NBUF; ++b) fetch(b);
    wait_copies<(S::NBUF - 1) * (kNp + kNq)>();
  } else {
    fetch(0);
    place(0);
    fetch(1);
    wait_reads();
  }
  meet();
#pragma unroll
  for (int n = 0; n < kFrags; ++n) read_one(0, 0, n);
  for (int32_t s = 0; s < (int32_t)steps; s += 2) {
    step(0);
    if (s + 1 < (int32_t)steps) step(1);
  }
  wait_copies<0>();  // no copy outlives the block's LDS, or lands on the sums
  if constexpr (S::G == 1) {
    finish<T, EPI>(
        a, i0 + wi, j0 + wj, acc, [](int p) { return 16 * p; }, [](int q) { return 32 * q; });
  } else {
    // the groups' sums side by side, added in the groups' order
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem);
    const int lane = (int)threadIdx.x & 63, g = lane >> 4, l = lane & 15;
#pragma unroll
    for (int x = 0; x < kXi; ++x)
#pragma unroll
      for (int y = 0; y < kXj; ++y) {
        const int i = wi + 16 * x + l, j = wj + 32 * (y / 2) + 8 * g + 4 * (y % 2);
        *reinterpret_cast<f32x4*>(sums + (group * S::kI + i) * S::kSumLd + j) = acc[x][y];
      }
    __syncthreads();
    constexpr int kEights = S::kI * S::kJ / 8;
    static_assert(kEights % 64 == 0, "whole waves");
#pragma unroll 1
    for (int t = (int)threadIdx.x; t < kEights; t += S::kThreads) {
      const int i = t / (S::kJ / 8), j = t % (S::kJ / 8) * 8;
      const int64_t gi = i0 + i, gj = j0 + j;
      Side<T, EPI> side;
      ColumnSide<T, EPI> column;
      if (a.splits == 1) {
        column_load<T, EPI>(a, gj, column);
        side_load<T, EPI>(a, gi, gj, side);
      }
      float v[8] = {};
#pragma unroll
      for (int k = 0; k < S::G; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(sums + (k * S::kI + i) * S::kSumLd + j + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * h + e] += x[e];
        }
      if (a.splits > 1) {
        const int64_t ld = (a.j + 7) & ~(int64_t)7;
        if (gi < a.i && gj < ld) El<float>::store8(a.partial + ((int64_t)blockIdx.y * a.i + gi) * ld + gj, v);
      } else {
        epilogue8<T, EPI, 1, 2>(a, gi, gj, v, column, side);
      }
    }
  }
}

// ---------------------------------------------------------------- few rows
// A layer over a few rows (the next tokens of a few sequences) is bound by reading W once.  A wave reads 1 KB of a row
// of W an instruction, whatever its alignment (a matrix fragment's 64 bytes of 16 rows streamed a fifth slower, and at
// half the rate off 16-byte rows), multiplies it with the same 1 KB of each row of x on the vector units, and adds its
// lanes' sums at the end.  A block's eight waves take JB rows of W, four a wave, and share out r where that leaves
// waves over.  1 x 14336 x 4096 takes 23.6 us, 5.0 TB/s of W, 1 x 4096 x 14336 20.3 us,
// 5.8 TB/s, with W's loads nontemporal: it is read once (24.2 us and 22.9 us without; where W lies in a cache, 1 x 2048 x
// 2048 4.49 us and 4.43 us without).
constexpr int kRowsWaves = 8, kRowsEach = 4, kMaxRows = 8;

template <typename T>
__device__ __forceinline__ float dot_chunk(const u32x4& w, const u32x4& x, float sum) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (El<T>::kBytes == 4) {
      sum = __builtin_fmaf(__uint_as_float(w[e]), __uint_as_float(x[e]), sum);
    } else {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const uint32_t we = w[e], xe = x[e];  // a bit cast of a vector's element itself takes the first one
      sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, we), __builtin_bit_cast(bf16x2, xe), sum, false);
    }
  }
  return sum;
}

template <typename T, int M, int JB>
__global__ __launch_bounds__(64 * kRowsWaves) void k_linear_rows(LinArgs a) {
  using Mem = typename El<T>::Mem;
  constexpr int kChunk = 16 / El<T>::kBytes, kGroups = kRowsWaves * kRowsEach / JB, kValues = kRowsEach * M;
  constexpr int kStep = 64 * kChunk, kAhead = M <= 2 ? 4 : 2;
  __shared__ float sums[kGroups][M][JB + 4];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63;
  const int group = wave % kGroups, jrow = wave / kGroups * kRowsEach;
  const int64_t j0 = (int64_t)blockIdx.x * JB, r = a.prod[0].r;
  // this thread's part of the epilogue, its loads under way from the start
  constexpr int kFinish = M * JB / 8;
  const int fi = (int)threadIdx.x / (JB / 8), fj = (int)threadIdx.x % (JB / 8) * 8;
  Side<T, kEpiLayer> side;
  ColumnSide<T, kEpiLayer> column;
  if (threadIdx.x < kFinish) {
    column_load<T, kEpiLayer>(a, j0 + fj, column);
    side_load<T, kEpiLayer>(a, fi, j0 + fj, side);
  }
  // rows past the last of W and x repeat it; what they give is not kept
  const Mem *w[kRowsEach], *x[M];
#pragma unroll
  for (int y = 0; y < kRowsEach; ++y) {
    const int64_t row = j0 + jrow + y;
    w[y] = static_cast<const Mem*>(a.prod[0].q) + (row < a.j ? row : a.j - 1) * a.prod[0].ldq;
  }
#pragma unroll
  for (int m = 0; m < M; ++m) x[m] = static_cast<const Mem*>(a.prod[0].p) + (m < a.i ? m : a.i - 1) * a.prod[0].ldp;
  float sum[kValues] = {};
  const auto run = [&](auto count, int64_t k0) {
    constexpr int kCount = decltype(count)::value;
    u32x4 cw[kCount][kRowsEach], cx[kCount][M];
#pragma unroll
    for (int u = 0; u < kCount; ++u) {
      const int64_t at = k0 + (int64_t)u * kGroups * kStep + lane * kChunk;
#pragma unroll
      for (int y = 0; y < kRowsEach; ++y) cw[u][y] = __builtin_nontemporal_load(reinterpret_cast<const typename El<T>::vec_mem*>(w[y] + at));
#pragma unroll
      for (int m = 0; m < M; ++m) cx[u][m] = *reinterpret_cast<const typename El<T>::vec_mem*>(x[m] + at);
    }
#pragma unroll
    for (int u = 0; u < kCount; ++u)
#pragma unroll
      for (int y = 0; y < kRowsEach; ++y)
#pragma unroll
        for (int m = 0; m < M; ++m) sum[y * M + m] = dot_chunk<T>(cw[u][y], cx[u][m], sum[y * M + m]);
  };
  int64_t k = (int64_t)group * kStep;
  constexpr int64_t kRound = (int64_t)kGroups * kStep;
  for (; k + (kAhead - 1) * kRound + kStep <= r; k += kAhead * kRound) run(std::integral_constant<int, kAhead>(), k);
  for (; k + kStep <= r; k += kRound) run(std::integral_constant<int, 1>(), k);
  if (k < r) {  // what is left, less than 1 KB
    const int64_t at = k + lane * kChunk, left = r - at;
    const int32_t valid = (int32_t)(left < 0 ? 0 : left < kChunk ? left : kChunk);
    u32x4 cx[M];
#pragma unroll
    for (int m = 0; m < M; ++m) cx[m] = load_chunk<T>(x[m] + at, valid);
#pragma unroll
    for (int y = 0; y < kRowsEach; ++y) {
      const u32x4 cw = load_chunk<T>(w[y] + at, valid);
#pragma unroll
      for (int m = 0; m < M; ++m) sum[y * M + m] = dot_chunk<T>(cw, cx[m], sum[y * M + m]);
    }
  }
  // the lanes' sums: while there are several values a lane exchanges half of them for its partner's other half, so
  // the values are dealt to the lanes as they are added; then the one left is added over the remaining lane bits
  int count = kValues;
#pragma unroll
  for (int bit = 32; bit > 0; bit >>= 1) {
    if (count > 1) {
      count /= 2;
#pragma unroll
      for (int v = 0; v < kValues / 2; ++v) {
        if (v < count) {
          const float low = sum[v], high = sum[v + count];
          sum[v] = ((lane & bit) ? high : low) + __shfl_xor((lane & bit) ? low : high, bit);
        }
      }
    } else {
      sum[0] += __shfl_xor(sum[0], bit);
    }
  }
  constexpr int kLanes = 64 / kValues;  // lanes with the same value
  if (lane % kLanes == 0) {
    const int v = lane / kLanes;
    sums[group][v % M][jrow + v / M] = sum[0];
  }
  __syncthreads();
  if (threadIdx.x >= kFinish) return;
  float v[8] = {};
#pragma unroll
  for (int g = 0; g < kGroups; ++g)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += sums[g][fi][fj + e];
  epilogue8<T, kEpiLayer, 1, 2>(a, fi, j0 + fj, v, column, side);
}

// Joins the partial sums in their order and applies the epilogue: eight j a thread.  Bound by memory: two ranges of
// 4096 x 2048 take 14 us, 6.2 TB/s.
template <typename T, int EPI>
__global__ __launch_bounds__(256) void k_linear_join(LinArgs a) {
  const int64_t eights = ((a.j + kCkptBlock - 1) / kCkptBlock) * 4, ld = (a.j + 7) & ~(int64_t)7;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = t / eights, j = (t - i * eights) * 8;
  float v[8] = {};
  if (i < a.i && j < ld) {
    for (int32_t s = 0; s < a.splits; ++s) {
      float x[8];
      El<float>::load8(a.partial + ((int64_t)s * a.i + i) * ld + j, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
  }
  Side<T, EPI> s;
  ColumnSide<T, EPI> c;
  column_load<T, EPI>(a, j, c);
  side_load<T, EPI>(a, i, j, s);
  epilogue8<T, EPI, 1, 2>(a, i, j, v, c, s);
}

// ---------------------------------------------------------------- copies on 16-byte rows
// Operands off 16-byte rows, copied to rows of whole 16 bytes with zeros at their ends: every chunk is read once at its
// element's address and written once, at about 5 TB/s.  A block takes kPackChunks of one operand.
constexpr int kPackChunks = 1024;
struct PackJob {
  const void* from;
  void* to;
  int64_t ld, run, across, chunks;  // chunks a row, and in all
  int64_t rows_on, chunks_on;       // from a thread's chunk to its next, 256 further
  uint32_t end;                     // the first block after this operand's
};
struct PackJobs {
  PackJob job[4];
  int32_t count;
  uint32_t blocks;
};

template <typename T>
__global__ __launch_bounds__(256) void k_pack(PackJobs jobs) {
  using Mem = typename El<T>::Mem;
  constexpr int kChunk = 16 / El<T>::kBytes;
  int k = 0;
  while (k + 1 < jobs.count && blockIdx.x >= jobs.job[k].end) ++k;
  const PackJob& j = jobs.job[k];
  const int64_t first = (int64_t)(blockIdx.x - (k ? jobs.job[k - 1].end : 0u)) * kPackChunks + threadIdx.x;
  const int64_t row0 = first / j.across;
  int64_t row = row0, c = first - row0 * j.across;
  u32x4 x[kPackChunks / 256];
#pragma unroll
  for (int u = 0; u < kPackChunks / 256; ++u) {
    const int64_t left = j.run - c * kChunk;
    if (first + u * 256 < j.chunks)
      x[u] = load_chunk<T>(static_cast<const Mem*>(j.from) + row * j.ld + c * kChunk, (int32_t)(left < kChunk ? left : kChunk));
    row += j.rows_on;
    c += j.chunks_on;
    if (c >= j.across) {
      c -= j.across;
      ++row;
    }
  }
#pragma unroll
  for (int u = 0; u < kPackChunks / 256; ++u)
    if (first + u * 256 < j.chunks) static_cast<u32x4*>(j.to)[first + u * 256] = x[u];
}

// ---------------------------------------------------------------- column sums
// A block sums COLS columns over all rows: COLS / 8 lanes hold a row's, and the sums are added through LDS in the
// rows' order, so one launch and no workspace do.  Bound by memory where there are enough columns (8192 x 14336 bf16
// takes 49 us with dy in HBM, 4.8 TB/s, 40 us with the same dy in every call, and adds 44 us to a weight gradient), else by
// how much its few blocks keep in flight: 32 columns a block there (1999 x 2048 6.2 us, with 64 columns a block 9.5).  Blocks
// of 32 bf16 columns read half cache lines, which costs where memory is the bound.
constexpr int kSumThreads = 1024;

template <typename T, int COLS>
__global__ __launch_bounds__(kSumThreads) void k_column_sum(const typename El<T>::Mem* __restrict__ dy, int64_t ld,
                                                            int64_t rows, int64_t cols,
                                                            typename El<T>::Mem* __restrict__ db) {
  constexpr int kLanes = COLS / 8, kRows = kSumThreads / kLanes, kParts = kSumThreads / COLS, kEach = kRows / kParts,
                kAhead = 4;
  __shared__ float s[kRows][COLS + 1];
  const int sub = (int)threadIdx.x / kLanes, c = (int)threadIdx.x % kLanes * 8;
  const int64_t j0 = wide_block() * COLS + c, valid = cols - j0;
  float v[8] = {};
  if (valid >= 8) {
    // kAhead rows' loads together; past the last row they repeat it and add nothing
    for (int64_t r0 = sub; r0 < rows; r0 += kAhead * kRows) {
      Raw8<T> x[kAhead];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int64_t r = r0 + n * kRows;
        x[n].load(dy + (r < rows ? r : rows - 1) * ld + j0);
      }
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        float u[8];
        x[n].get(u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r0 + n * kRows < rows ? u[e] : 0.f;
      }
    }
  } else if (valid > 0) {
#pragma unroll 4
    for (int64_t r = sub; r < rows; r += kRows) {
      float x[8];
      load_row8<T>(dy + r * ld + j0, valid, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s[sub][c + e] = v[e];
  __syncthreads();
  // kParts threads a column add kEach rows each, then one thread their sums
  const int col = (int)threadIdx.x % COLS, part = (int)threadIdx.x / COLS;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < kEach; ++k) sum += s[part * kEach + k][col];
  __syncthreads();
  s[part][col] = sum;
  __syncthreads();
  const int64_t j = wide_block() * COLS + col;
  if (part == 0 && j < cols) {
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < kParts; ++k) sum += s[k][col];
    El<T>::store(db + j, sum);
  }
}

// ---------------------------------------------------------------- launches
namespace {
template <typename F>
void with_element(int dtype, F&& fn) {
  if (dtype == 1)
    fn(Bf16());
  else
    fn(float());
}
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int kComputeUnits = 256;

// The first row stride whose tiles cannot be copied to LDS directly: copies take 32-bit offsets from a tile's first
// byte, and those past 0x7FFFFFF0 read as zeros.  A tile has up to 256 bf16 or 128 fp32 rows of a direct operand
// (510 ld bytes), and a stage 64 bf16 or 32 fp32 of a transposed one (126 ld bytes and a tile's 512).
constexpr int64_t wide_ld(bool trans) { return trans ? (int64_t)1 << 24 : (int64_t)1 << 22; }

// Whether an operand's stages can be copied to LDS directly: 16-byte rows, and no wide ones.
bool operand_fits(const void* p, int64_t ld, int64_t r, bool trans, int bytes) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * bytes % 16 == 0 && (trans || r * bytes % 16 == 0) &&
         ld < wide_ld(trans);
}

// fn(element type, P transposed, Q transposed, epilogue) of an operation.
template <typename F>
void with_form(int dtype, LinEpilogue epi, F&& fn) {
  with_element(dtype, [&](auto t) {
    if (epi == kEpiLayer)
      fn(t, std::false_type(), std::false_type(), std::integral_constant<int, kEpiLayer>());
    else if (epi == kEpiDgrad)
      fn(t, std::false_type(), std::true_type(), std::integral_constant<int, kEpiDgrad>());
    else
      fn(t, std::true_type(), std::true_type(), std::integral_constant<int, kEpiStore>());
  });
}
}  // namespace

namespace {
// The tiles a product can be computed with.
enum TileForm : int32_t { kFast = 1, kMiddle = 2, kSmall = 3, kTiny = 4, kRows = 5, kNarrow = 6, kPair = 7 };
using MiddleShape = GroupShape<64, 64, 2, 2, 1, 2>;  // 128 x 128, two blocks a compute unit
using PairShape = GroupShape<64, 64, 2, 2, 2, 2>;     // 128 x 128, r in two
using SmallShape = GroupShape<64, 64, 1, 1, 4, 2>;   // 64 x 64, r in four
using NarrowShape = GroupShape<32, 64, 1, 1, 4, 3>;  // 32 x 64, r in four
using TinyShape = GroupShape<16, 32, 1, 1, 4, 3>;    // 16 x 32, r in four, two blocks a compute unit

// What the choice of a tile goes by: the tile, blocks that run together on a compute unit, stages of r that a block
// takes together (its groups), and measured microseconds: of a stage with as many blocks on each unit, of one with one
// block a unit, and of a block's start and end.
struct FormCost {
  int32_t form, i, j, threads, resident, groups;
  double stage, alone, rest;
};
template <typename S>
constexpr FormCost cost(int32_t form, double stage, double alone, double rest) {
  return {form, S::kI, S::kJ, S::kThreads, S::kResident, S::G, stage, alone, rest};
}
// bf16 with stages copied to LDS directly, by how many operands are transposed; the same by way of registers, where
// the other tiles are slower than these at every size tried (64 x 64, one wave a SIMD, twice as long); fp32 both ways,
// whose matrix instructions take 16 times as long.
constexpr FormCost direct_fast(double stage) { return {kFast, kFastB, kFastB, kFastThreads, 1, 1, stage, stage, 10.0}; }
const FormCost kDirectCosts[3][6] = {
    {direct_fast(1.40), cost<MiddleShape>(kMiddle, 0.90, 0.66, 6.0), cost<SmallShape>(kSmall, 0.92, 0.92, 5.2),
     cost<NarrowShape>(kNarrow, 0.55, 0.55, 5.0), cost<TinyShape>(kTiny, 0.45, 0.28, 4.2),
     cost<PairShape>(kPair, 0.95, 0.95, 7.2)},
    {direct_fast(1.43), cost<MiddleShape>(kMiddle, 0.92, 0.66, 6.0), cost<SmallShape>(kSmall, 0.90, 0.90, 5.2),
     cost<NarrowShape>(kNarrow, 0.58, 0.58, 5.0), cost<TinyShape>(kTiny, 0.50, 0.30, 4.2),
     cost<PairShape>(kPair, 0.95, 0.95, 7.2)},
    {direct_fast(1.46), cost<MiddleShape>(kMiddle, 0.94, 0.70, 6.0), cost<SmallShape>(kSmall, 0.92, 0.92, 5.2),
     cost<NarrowShape>(kNarrow, 0.60, 0.60, 5.0), cost<TinyShape>(kTiny, 0.60, 0.60, 4.2),
     cost<PairShape>(kPair, 0.95, 0.95, 7.2)}};
const FormCost kStagedCosts[3][2] = {{cost<MiddleShape>(kMiddle, 1.15, 1.02, 9.0), cost<TinyShape::Staged>(kTiny, 0.8, 0.6, 6.5)},
                                     {cost<MiddleShape>(kMiddle, 1.31, 1.45, 9.0), cost<TinyShape::Staged>(kTiny, 0.8, 0.6, 6.5)},
                                     {cost<MiddleShape>(kMiddle, 1.74, 1.57, 9.0), cost<TinyShape::Staged>(kTiny, 1.3, 1.0, 6.5)}};
const FormCost kFp32Costs[] = {cost<MiddleShape>(kMiddle, 3.95, 2.1, 7.0), cost<SmallShape>(kSmall, 2.35, 2.35, 4.5),
                               cost<TinyShape>(kTiny, 0.6, 0.32, 4.5)};
const FormCost kFp32StagedCosts[] = {cost<MiddleShape>(kMiddle, 4.65, 2.5, 7.0), cost<TinyShape::Staged>(kTiny, 1.2, 0.75, 5.0)};

// The kernel for few rows of x: its start, and the bytes a microsecond that it reads with 1, 2, 4 and 8 rows of bf16 (fp32
// is chosen by the same: 14336 x 4096 takes 45 us with 1 or 2 rows, 52 with 5 or 8, 5.2 and 4.5 TB/s).  Against
// 16 x 32 tiles with 5 rows: 14336 x 4096 31.5 us (23.6), 4096 x 4096 10.2 (9.8), 2048 x 2048 5.6 (6.2), 960 x 4096 7.0
// (7.7); with 3 rows 25.6 (23.4), 8.8 (9.8), 4.8 (6.2) and 5.0 (7.7).
constexpr double kRowsStart = 3.5, kRowsRate[4] = {5.8e6, 5.6e6, 4.9e6, 3.8e6};

// A product's sizes as the choice sees them: of out, its stages of r, and the microseconds that 65,536 values' epilogue
// keeps a compute unit's vector units busy.
struct Sizes {
  int64_t i, j, stages;
  double epilogue;
  double bytes;  // of the operands
  int64_t line;  // columns of a transposed Q in a cache line, or 0
};

// Microseconds of `splits` ranges of r with tile f, or kNever where its grid cannot be launched.
constexpr double kNever = 1e30;
double time_of(const FormCost& f, const Sizes& z, int64_t splits) {
  const int64_t tiles = div_up(z.i, f.i) * div_up(z.j, f.j), blocks = tiles * splits;
  const int64_t slots = (int64_t)kComputeUnits * f.resident;
  if (tiles > kMaxThreads / f.threads) return kNever;
  const int64_t rounds = blocks / slots, left = blocks % slots;
  const double steps = (double)div_up(z.stages, splits * f.groups);
  const double end = splits > 1 ? 0.0 : z.epilogue * (double)(f.i * f.j) / 65536.0;
  const double full = f.rest + steps * f.stage + end * f.resident;
  double us = (double)rounds * full;
  // a part of a round: fewer units run two epilogues (512 x 8960 x 1536, gated: 37 us in 280 tiles of 128 x 128, 42 us in
  // three ranges of r of 256 x 256)
  if (left > kComputeUnits)
    us += f.rest + steps * f.stage + end * f.resident * (double)left / (double)slots;
  else if (left)
    us += rounds ? full : f.rest + steps * f.alone + end;
  // Memory delivers the operands at 5.6 TB/s after a start of 4.5 us, and to a block at 40 GB/s, half of it where the
  // block takes half of each cache line (32 x 4096 x 14336 with W read along its rows: 51 us in 128 tiles of 16 x 32,
  // 31 us in 256 blocks of 32 x 64); between tiles that it bounds, the one with the least work.
  const double rate = (f.j < z.line ? 20e3 : 40e3) * (double)blocks;
  const double memory = 4.5 + z.bytes / (rate < 5.6e6 ? rate : 5.6e6);
  double sum = (us > memory ? us : memory) + 0.1 * us;
  // the partial sums are written and read, and another launch joins them
  if (splits > 1) sum += 2.0 + (double)splits * (double)z.i * (double)z.j * 8.0 / 8e6;
  return sum;
}

// The least-time tile and number of ranges of r by those costs.  Ranges beyond one block a place only cost.
double choose(const FormCost* costs, int count, const Sizes& z, LinPart& part) {
  double least = kNever;
  part = {z.i, 0, 1};
  for (int c = 0; c < count; ++c) {
    const FormCost& f = costs[c];
    const int64_t tiles = div_up(z.i, f.i) * div_up(z.j, f.j), slots = (int64_t)kComputeUnits * f.resident;
    int64_t most = slots / tiles + 1;
    if (most > 16) most = 16;
    if (most > z.stages / (2 * f.groups)) most = z.stages / (2 * f.groups);
    for (int64_t splits = 1; splits == 1 || splits <= most; ++splits) {
      const double us = time_of(f, z, splits);
      if (us < least) {
        least = us;
        part = {z.i, f.form, (int32_t)splits};
      }
    }
  }
  return least;
}

// The same in one launch or two: rounds of blocks that fill every compute unit, then the rows that are left with the
// tile that suits them, where that beats a last round of few blocks.  (4096 x 8960 x 1536 with a gated epilogue: three
// rounds of 256 x 256 tiles, the last of 48, take 193 us, two rounds and the rest 179 us.)
double choose_parts(const FormCost* costs, int count, const Sizes& z, LinPlan& plan) {
  constexpr double kWorthIt = 15.0, kLaunch = 2.0;
  double least = choose(costs, count, z, plan.part[0]);
  plan.parts = 1;
  if (least < kWorthIt) return least;
  for (int c = 0; c < count; ++c) {
    const FormCost& f = costs[c];
    const int64_t across = div_up(z.j, f.j), slots = (int64_t)kComputeUnits * f.resident;
    const int64_t rounds = div_up(z.i, f.i) * across / slots, rows = rounds * slots / across * f.i;
    if (rows <= 0 || rows >= z.i) continue;
    Sizes first = z, rest = z;
    first.i = rows;
    rest.i = z.i - rows;
    LinPart other;
    const double us = time_of(f, first, 1) + kLaunch + choose(costs, count, rest, other);
    if (us < least) {
      least = us;
      plan.part[0] = {rows, f.form, 1};
      plan.part[1] = other;
      plan.parts = 2;
    }
  }
  return least;
}

// An operand as it lies in memory: `rows` runs of `run` elements.
struct Operand {
  const void* p;
  int64_t ld, rows, run;
  bool fits, trans;
};
// Operands 2 s and 2 s + 1 are P and Q of product s.
void operands(const LinArgs& a, LinEpilogue epi, int bytes, Operand (&o)[4]) {
  const bool pt = epi == kEpiStore, qt = epi != kEpiLayer;
  for (int s = 0; s < 2; ++s) {
    const LinProduct& pr = a.prod[s];
    o[2 * s] = {pr.p, pr.ldp, pt ? pr.r : a.i, pt ? a.i : pr.r, pr.r == 0 || operand_fits(pr.p, pr.ldp, pr.r, pt, bytes), pt};
    o[2 * s + 1] = {pr.q, pr.ldq, qt ? pr.r : a.j, qt ? a.j : pr.r, pr.r == 0 || operand_fits(pr.q, pr.ldq, pr.r, qt, bytes), qt};
  }
}
int64_t packed_ld(int64_t run, int bytes) { return div_up(run * bytes, 16) * 16 / bytes; }
}  // namespace

LinPlan linear_plan(const LinArgs& a, int dtype, LinEpilogue epi) {
  const int bytes = dtype == 1 ? 2 : 4;
  const int64_t deep = 128 / bytes;
  LinPlan best{};
  Sizes z{a.i, a.j, div_up(a.prod[0].r, deep) + div_up(a.prod[1].r, deep), 0.0, 0.0, epi == kEpiLayer ? 0 : 128 / bytes};
  if (epi == kEpiLayer) z.epilogue = (a.act ? 8.0 : 0.0) + (a.codes ? 6.0 : 0.0) + (a.mul ? 2.0 : 0.0) + (a.residual ? 2.0 : 0.0);
  if (epi == kEpiDgrad) z.epilogue = a.up_codes ? 22.0 : a.z_codes ? 13.0 : 0.0;
  Operand o[4];
  operands(a, epi, bytes, o);
  int32_t off = 0;  // operands that cannot be copied to LDS directly as they lie
  bool wide = false;  // one of them is too wide for direct copies even where it is packed
  double moved = 0.0;
  for (int k = 0; k < 4; ++k) z.bytes += (double)o[k].rows * (double)o[k].run * bytes;
  for (int k = 0; k < 4; ++k)
    if (!o[k].fits) {
      off |= 1 << k;
      wide |= packed_ld(o[k].run, bytes) >= wide_ld(o[k].trans);
      moved += 2.0 * (double)o[k].rows * (double)o[k].run * bytes;
    }
  const int transposed = epi == kEpiStore ? 2 : epi == kEpiDgrad ? 1 : 0;  // operands
  const double direct = dtype == 1 ? choose_parts(kDirectCosts[transposed], 6, z, best) : choose_parts(kFp32Costs, 3, z, best);
  double least = direct;
  best.direct = 1;
  if (off) {
    // copies on 16-byte rows first, or stages by way of registers: a launch and the bytes against slower stages
    LinPlan staged{};
    const double through = dtype == 1 ? choose_parts(kStagedCosts[transposed], 2, z, staged) : choose_parts(kFp32StagedCosts, 2, z, staged);
    least = direct + 6.0 + moved / 5.0e6;
    if (wide || through <= least) {
      best = staged;
      least = through;
    } else {
      best.pack = off;
    }
  }
  // few rows: the kernel that takes operands of any alignment without a copy (16 threads a column where there are many)
  if (epi == kEpiLayer && a.i <= kMaxRows && a.j <= kMaxThreads / 16 - 32) {
    const double rate = kRowsRate[a.i > 4 ? 3 : a.i > 2 ? 2 : a.i - 1];
    if (kRowsStart + z.bytes / rate <= least) {
      best = LinPlan{};
      best.part[0] = {a.i, kRows, 1};
      best.parts = 1;
    }
  }
  // the parts run one after the other and share the place of their partial sums
  for (int p = 0; p < best.parts; ++p) {
    const LinPart& q = best.part[p];
    const size_t sums = q.splits > 1 ? (size_t)q.splits * (size_t)q.rows * (size_t)(div_up(a.j, 8) * 8) * 4 : 0;
    if (sums > best.workspace) best.workspace = sums;
  }
  for (int k = 0; k < 4; ++k)
    if (best.pack >> k & 1) {
      best.packed[k] = best.workspace;
      best.workspace += (size_t)o[k].rows * (size_t)packed_ld(o[k].run, bytes) * bytes;
    }
  return best;
}

namespace {
template <typename S, typename T, bool PT, bool QT, int EPI>
hipError_t launch_group(const LinArgs& a, bool direct, hipStream_t stream) {
  const dim3 grid((uint32_t)(div_up(a.i, S::kI) * div_up(a.j, S::kJ)), (uint32_t)a.splits);
  if (direct) {
    k_linear_group<T, PT, QT, EPI, S, true><<<grid, dim3(S::kThreads), S::kLds, stream>>>(a);
  } else if constexpr (std::is_same<S, MiddleShape>::value || std::is_same<S, TinyShape>::value) {
    using R = typename S::Staged;
    k_linear_group<T, PT, QT, EPI, R, false><<<grid, dim3(R::kThreads), R::kLds, stream>>>(a);
  } else {
    return hipErrorInvalidConfiguration;
  }
  return hipGetLastError();
}
}  // namespace

namespace {
const void* skip_bytes(const void* p, int64_t bytes) { return p ? static_cast<const char*>(p) + bytes : p; }
void* skip_bytes(void* p, int64_t bytes) { return p ? static_cast<char*>(p) + bytes : p; }

// Rows [from, from + rows) of a product.
LinArgs rows_of(LinArgs a, int64_t from, int64_t rows, int bytes, bool pt) {
  const int64_t nb = ckpt_blocks(a.j);
  for (LinProduct& pr : a.prod)
    if (pr.r > 0) pr.p = skip_bytes(pr.p, (pt ? from : from * pr.ldp) * bytes);
  a.i = rows;
  a.out = skip_bytes(a.out, from * a.ldout * bytes);
  a.mul = skip_bytes(a.mul, from * a.ldmul * bytes);
  a.residual = skip_bytes(a.residual, from * a.ldres * bytes);
  a.out_up = skip_bytes(a.out_up, from * a.ldup * bytes);
  a.codes = static_cast<int8_t*>(skip_bytes(a.codes, from * nb * kCkptBlock));
  a.exps = static_cast<uint8_t*>(skip_bytes(a.exps, from * nb));
  a.z_codes = static_cast<const int8_t*>(skip_bytes(a.z_codes, from * nb * kCkptBlock));
  a.z_exps = static_cast<const uint8_t*>(skip_bytes(a.z_exps, from * nb));
  a.up_codes = static_cast<const int8_t*>(skip_bytes(a.up_codes, from * nb * kCkptBlock));
  a.up_exps = static_cast<const uint8_t*>(skip_bytes(a.up_exps, from * nb));
  return a;
}

template <typename T>
hipError_t launch_rows(const LinArgs& a, hipStream_t stream) {
  // a checkpoint's blocks need 32 columns; without one narrower blocks until there are enough of them
  const auto launch = [&](auto jb) {
    const dim3 grid((uint32_t)div_up(a.j, jb())), block(64 * kRowsWaves);
    if (a.i == 1)
      k_linear_rows<T, 1, jb()><<<grid, block, 0, stream>>>(a);
    else if (a.i == 2)
      k_linear_rows<T, 2, jb()><<<grid, block, 0, stream>>>(a);
    else if (a.i <= 4)
      k_linear_rows<T, 4, jb()><<<grid, block, 0, stream>>>(a);
    else
      k_linear_rows<T, 8, jb()><<<grid, block, 0, stream>>>(a);
  };
  if (a.codes || a.j >= 32 * kComputeUnits)
    launch(std::integral_constant<int, 32>());
  else if (a.j >= 16 * kComputeUnits)
    launch(std::integral_constant<int, 16>());
  else
    launch(std::integral_constant<int, 8>());
  return hipGetLastError();
}
}  // namespace

hipError_t launch_linear(const LinArgs& args, int dtype, LinEpilogue epi, const LinPlan& plan, void* workspace,
                         hipStream_t stream) {
  const int bytes = dtype == 1 ? 2 : 4;
  LinArgs whole = args;
  whole.partial = static_cast<float*>(workspace);
  hipError_t e = hipSuccess;
  if (plan.pack) {
    PackJobs jobs{};
    Operand o[4];
    operands(whole, epi, bytes, o);
    for (int k = 0; k < 4; ++k)
      if (plan.pack >> k & 1) {
        void* to = static_cast<char*>(workspace) + plan.packed[k];
        const int64_t ld = packed_ld(o[k].run, bytes), across = ld * bytes / 16;
        PackJob& j = jobs.job[jobs.count++];
        j = {o[k].p, to, o[k].ld, o[k].run, across, o[k].rows * across, 256 / across, 256 % across};
        jobs.blocks += (uint32_t)div_up(j.chunks, kPackChunks);
        j.end = jobs.blocks;
        LinProduct& pr = whole.prod[k / 2];
        (k % 2 ? pr.q : pr.p) = to;
        (k % 2 ? pr.ldq : pr.ldp) = ld;
      }
    if (jobs.blocks > kMaxThreads / 256) return hipErrorInvalidConfiguration;
    with_element(dtype, [&](auto t) { k_pack<decltype(t)><<<dim3(jobs.blocks), dim3(256), 0, stream>>>(jobs); });
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  int64_t from = 0;
  for (int p = 0; p < plan.parts && e == hipSuccess; ++p) {
    const LinPart& part = plan.part[p];
    LinArgs a = rows_of(whole, from, part.rows, bytes, epi == kEpiStore);
    a.splits = part.splits;
    from += part.rows;
    const int64_t eights = a.i * ckpt_blocks(a.j) * 4;  // of the join
    if (part.form == 0 || (a.splits > 1 && eights > kMaxThreads - 256)) return hipErrorInvalidConfiguration;
    with_form(dtype, epi, [&](auto t, auto pt, auto qt, auto ep) {
      using T = decltype(t);
      if constexpr (std::is_same<T, Bf16>::value) {
        if (part.form == kFast) {
          const dim3 grid((uint32_t)(div_up(a.i, kFastB) * div_up(a.j, kFastB)), (uint32_t)a.splits);
          k_linear_fast<pt(), qt(), ep()><<<grid, dim3(kFastThreads), 8 * kHalfBytes, stream>>>(a);
          e = hipGetLastError();
        }
      }
      if constexpr (ep() == kEpiLayer) {
        if (part.form == kRows) e = launch_rows<T>(a, stream);
      }
      if (part.form == kMiddle) e = launch_group<MiddleShape, T, pt(), qt(), ep()>(a, plan.direct, stream);
      if (part.form == kSmall) e = launch_group<SmallShape, T, pt(), qt(), ep()>(a, plan.direct, stream);
      if constexpr (std::is_same<T, Bf16>::value) {
        if (part.form == kPair) e = launch_group<PairShape, T, pt(), qt(), ep()>(a, plan.direct, stream);
        if (part.form == kNarrow) e = launch_group<NarrowShape, T, pt(), qt(), ep()>(a, plan.direct, stream);
      }
      if (part.form == kTiny) e = launch_group<TinyShape, T, pt(), qt(), ep()>(a, plan.direct, stream);
      if (e != hipSuccess || a.splits <= 1) return;
      k_linear_join<T, ep()><<<dim3((uint32_t)div_up(eights, 256)), dim3(256), 0, stream>>>(a);
      e = hipGetLastError();
    });
  }
  return e;
}

hipError_t launch_column_sum(const void* dy, int64_t ld, int64_t rows, int64_t cols, int dtype, void* db,
                             hipStream_t stream) {
  with_element(dtype, [&](auto t) {
    using T = decltype(t);
    using Mem = typename El<T>::Mem;
    const auto launch = [&](auto n) {
      k_column_sum<T, n()><<<wide_grid(div_up(cols, n())), dim3(kSumThreads), 0, stream>>>(
          static_cast<const Mem*>(dy), ld, rows, cols, static_cast<Mem*>(db));
    };
    if (cols >= 32 * kComputeUnits)
      launch(std::integral_constant<int, 64>());
    else
      launch(std::integral_constant<int, 32>());
  });
  return hipGetLastError();
}

}  // namespace smat
