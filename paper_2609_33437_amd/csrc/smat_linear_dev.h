// Device pieces of the linear-layer kernels: activations, checkpoint blocks and epilogues on eight
// consecutive values of a row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "smat.h"
#include "smat_device.h"
#include "smat_linear.h"

namespace smat {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int64_t wide_block() { return ((int64_t)blockIdx.y << kWideShift) + blockIdx.x; }

// ---------------------------------------------------------------- element types
template <typename T>
struct El;
template <>
struct El<float> {
  using Mem = float;
  static constexpr int kBytes = 4;
  typedef u32x4 vec_mem __attribute__((aligned(4)));  // 16 bytes at any element's address
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  // eight elements at any element's address
  static __device__ __forceinline__ void load8(const float* p, float v[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4_mem*>(p), b = *reinterpret_cast<const f32x4_mem*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = a[e];
      v[4 + e] = b[e];
    }
  }
  static __device__ __forceinline__ void store8(float* p, const float v[8]) {
    *reinterpret_cast<f32x4_mem*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_mem*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};
template <>
struct El<Bf16> {
  using Mem = uint16_t;
  static constexpr int kBytes = 2;
  typedef u32x4 vec_mem __attribute__((aligned(2)));
  static __device__ __forceinline__ float load(const uint16_t* p) { return bf16_to_f32(*p); }
  static __device__ __forceinline__ void store(uint16_t* p, float v) { *p = to_bf16(v); }
  static __device__ __forceinline__ void load8(const uint16_t* p, float v[8]) {
    const u32x4 x = *reinterpret_cast<const vec_mem*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(x[e] << 16);
      v[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store8(uint16_t* p, const float v[8]) {
    *reinterpret_cast<vec_mem*>(p) =
        u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
};

// Elements [0, valid) of eight, zeros after them (valid may lie outside [0, 8]).
template <typename T>
__device__ __forceinline__ void load_row8(const typename El<T>::Mem* p, int64_t valid, float v[8]) {
  if (valid >= 8) {
    El<T>::load8(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < valid ? El<T>::load(p + e) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_row8(typename El<T>::Mem* p, int64_t valid, const float v[8]) {
  if (valid >= 8) {
    El<T>::store8(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < valid) El<T>::store(p + e, v[e]);
  }
}

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

// ---------------------------------------------------------------- sums over lanes
// What `op` makes of the values of N consecutive lanes (N = 4, 8, 16, 32 or 64), in each of them: neighbours are exchanged
// within 16 lanes by the vector unit's own lane operands, and rows of 16 by the swaps, where a shuffle would pass
// LDS six times.  op is symmetric, so all lanes form the same bits.
template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// op of this lane's value and that of lane l ^ 16, l ^ 32.
template <typename F>
__device__ __forceinline__ float with_lane16(float v, F&& op) {
  const uint32_t b = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename F>
__device__ __forceinline__ float with_lane32(float v, F&& op) {
  const uint32_t b = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int N, typename F>
__device__ __forceinline__ float over_lanes(float v, F&& op) {
  v = op(v, lane_move<0xB1>(v));                       // l ^ 1
  v = op(v, lane_move<0x4E>(v));                       // l ^ 2
  if constexpr (N > 4) v = op(v, lane_move<0x141>(v));  // 7 - l: the other four
  if constexpr (N > 8) v = op(v, lane_move<0x140>(v));  // 15 - l: the other eight
  if constexpr (N > 16) v = with_lane16(v, op);
  if constexpr (N > 32) v = with_lane32(v, op);
  return v;
}
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
  return over_lanes<N>(v, [](float a, float b) { return a + b; });
}
template <int N>
__device__ __forceinline__ float lanes_max(float v) {
  return over_lanes<N>(v, [](float a, float b) { return fmaxf(a, b); });
}

// ---------------------------------------------------------------- activations
// exp, erf and a reciprocal to the accuracy that the type of the result holds: the library's functions
// for fp32; for bf16 the hardware's exp2 and reciprocal, and erfc by formula 7.1.26 of Abramowitz and
// Stegun, "Handbook of Mathematical Functions" (absolute error at most 1.5e-7).
template <typename T>
__device__ __forceinline__ float act_exp(float x) {
  if constexpr (sizeof(typename El<T>::Mem) == 4)
    return expf(x);
  else
    return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
}
template <typename T>
__device__ __forceinline__ float act_rcp(float x) {
  if constexpr (sizeof(typename El<T>::Mem) == 4)
    return 1.f / x;
  else
    return __builtin_amdgcn_rcpf(x);
}
template <typename T>
__device__ __forceinline__ float logistic(float x) {
  return act_rcp<T>(1.f + act_exp<T>(-x));
}
// The logistic function and 1 minus it, without the subtraction's cancellation.  Where exp(-x) overflows the first is 0, as
// logistic() has it, and the second need only be finite: it stands beside a factor of the first.
template <typename T>
__device__ __forceinline__ void logistic_both(float x, float& g, float& h) {
  const float e = act_exp<T>(-x);
  g = act_rcp<T>(1.f + e);
  h = fminf(e, 1e38f) * g;
}
// The standard normal's distribution function at z, and exp(-z^2 / 2).  (The coefficients carry the half.)
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float& gauss) {
  if constexpr (sizeof(typename El<T>::Mem) == 4) {
    gauss = expf(-0.5f * z * z);
    return 0.5f * erfcf(-z * 0.70710678118654752440f);
  } else {
    gauss = act_exp<T>(-0.5f * z * z);
    const float x = fabsf(z) * 0.70710678118654752440f;
    const float t = act_rcp<T>(__builtin_fmaf(0.3275911f, x, 1.f));
    float p = __builtin_fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
    p = __builtin_fmaf(p, t, 0.5f * 1.421413741f);
    p = __builtin_fmaf(p, t, 0.5f * -0.284496736f);
    p = __builtin_fmaf(p, t, 0.5f * 0.254829592f);
    const float half_erfc = p * t * gauss;  // of |z| / sqrt(2)
    return z < 0.f ? half_erfc : 1.f - half_erfc;
  }
}
constexpr float kGeluTanhA = 0.79788456080286535588f, kGeluTanhB = 0.044715f;  // sqrt(2 / pi)

// act(z).  `act` is uniform over a launch.
template <typename T>
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == SMAT_ACT_SILU) return z * logistic<T>(z);
  if (act == SMAT_ACT_GELU_TANH)  // (1 + tanh t) / 2 is the logistic function of 2 t
    return z * logistic<T>(2.f * kGeluTanhA * (z + kGeluTanhB * z * z * z));
  if (act == SMAT_ACT_GELU) {
    float gauss;
    return z * normal_cdf<T>(z, gauss);
  }
  return z;
}

// act(z) and act'(z) of a finite or NaN z (what a checkpoint holds).  A NaN reaches both through z's product.
template <typename T>
__device__ __forceinline__ void act_both(float z, int act, float& value, float& slope) {
  if (act == SMAT_ACT_SILU) {
    float g, h;
    logistic_both<T>(z, g, h);
    value = z * g;
    slope = __builtin_fmaf(value, h, g);
  } else if (act == SMAT_ACT_GELU_TANH) {
    float g, h;
    logistic_both<T>(2.f * kGeluTanhA * (z + kGeluTanhB * z * z * z), g, h);
    value = z * g;
    // past |z| = 16 the logistic is 0 or 1 and the slope's second term is 0, however large z^2 grows
    const float zc = fminf(fmaxf(z, -16.f), 16.f);
    slope = __builtin_fmaf(value * h, 2.f * kGeluTanhA * __builtin_fmaf(3.f * kGeluTanhB * zc, zc, 1.f), g);
  } else if (act == SMAT_ACT_GELU) {
    float gauss;
    const float below = normal_cdf<T>(z, gauss);
    value = z * below;
    slope = __builtin_fmaf(z * 0.39894228040143267794f, gauss, below);
  } else {
    value = z;
    slope = 1.f;
  }
}

// ---------------------------------------------------------------- checkpoint blocks
// A block holds x_j = q_j 2^E with E = max(floor(log2 max|x|) - 6, -126) and q_j = rne(x_j 2^-E) held to
// +-127; its byte is E + 127.  The power of two is exact to multiply and divide by, and a code's seven
// bits fit bf16's eight, so reading back rounds nothing.  A block with a NaN or an infinity has byte 255
// and codes 0: the byte's 2^128 is an infinity, and 0 times it reads back as NaN.
//
// `bits`: max |x| of the block as an integer (NaN above infinity above every number).
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t ckpt_byte(uint32_t bits) {
  const int e = (int)(bits >> 23) - 6;
  return bits >= 0x7F800000u ? 255u : (uint32_t)(e > 1 ? e : 1);
}
// Codes of eight values.  Adding 1.5 * 2^23 rounds x 2^-E to nearest even and leaves the integer, in two's complement,
// in the low bits; held to +-127 there, its low byte is the code.
__device__ __forceinline__ u32x2 ckpt_pack8(const float v[8], uint32_t byte) {
  constexpr float kMagic = 12582912.f;
  constexpr int kMagicBits = 0x4B400000;
  const float inverse = __uint_as_float((254u - byte) << 23);  // 2^-E; unused for a block of byte 255
  u32x2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int bits = (int)__float_as_uint(__builtin_fmaf(v[4 * h + e], inverse, kMagic));
      q[e] = (uint32_t)min(max(bits, kMagicBits - 127), kMagicBits + 127);
    }
    const uint32_t lo = __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(q[3], q[2], 0x0C0C0400u);
    out[h] = byte == 255u ? 0u : lo | hi << 16;
  }
  return out;
}
__device__ __forceinline__ void ckpt_unpack8(u32x2 codes, uint32_t byte, float v[8]) {
  const float scale = __uint_as_float(byte << 23);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)((int)(codes[e / 4] << (24 - 8 * (e % 4))) >> 24) * scale;
}

// max over the four lanes that hold a block: lanes l ^ A, l ^ B, l ^ A ^ B.
template <int A, int B>
__device__ __forceinline__ uint32_t block_max(const float v[8]) {
  uint32_t m = abs_bits(v[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) m = max(m, abs_bits(v[e]));
  m = max(m, (uint32_t)__shfl_xor((int)m, A));
  return max(m, (uint32_t)__shfl_xor((int)m, B));
}

// ---------------------------------------------------------------- epilogues
// What an epilogue reads beside its eight values, as it lies in memory.  Loads of whole eights can be
// issued ahead of their use (side_load); at a row's end the epilogue loads what there is itself.
template <typename T>
struct Raw8;
template <>
struct Raw8<Bf16> {
  u32x4 x;
  __device__ __forceinline__ void load(const uint16_t* p) { x = *reinterpret_cast<const El<Bf16>::vec_mem*>(p); }
  // the first `valid` elements, zeros after them
  __device__ __forceinline__ void load_some(const uint16_t* p, int64_t valid) {
    x = load_chunk<Bf16>(p, (int32_t)(valid < 8 ? valid : 8));
  }
  __device__ __forceinline__ void get(float v[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(x[e] << 16);
      v[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u);
    }
  }
};
template <>
struct Raw8<float> {
  f32x4 x[2];
  __device__ __forceinline__ void load(const float* p) {
    x[0] = *reinterpret_cast<const f32x4_mem*>(p);
    x[1] = *reinterpret_cast<const f32x4_mem*>(p + 4);
  }
  __device__ __forceinline__ void load_some(const float* p, int64_t valid) {
    const int32_t n = (int32_t)(valid < 8 ? valid : 8);
    x[0] = __builtin_bit_cast(f32x4, load_chunk<float>(p, n < 4 ? n : 4));
    x[1] = __builtin_bit_cast(f32x4, load_chunk<float>(p + 4, n - 4));
  }
  __device__ __forceinline__ void get(float v[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e / 4][e % 4];
  }
};
template <typename T, int EPI>
struct Side {};
// The same of a column: it serves every row.
template <typename T, int EPI>
struct ColumnSide {};
template <typename T>
struct ColumnSide<T, kEpiLayer> {
  Raw8<T> bias;
};
template <typename T>
struct Side<T, kEpiLayer> {
  Raw8<T> mul, residual;
};
template <typename T>
struct Side<T, kEpiDgrad> {
  u32x2 z, up;
  uint32_t z_byte, up_byte;
};
template <typename T>
struct Side<T, kEpiXent> {
  int64_t target;
};
template <typename T>
struct Side<T, kEpiXentGrad> {
  int64_t target;
  float lse, low, scale;
};
template <typename T>
struct Side<T, kEpiSum> {
  Raw8<float> sum;
  int64_t row;  // of out; -1 - row: it is zeros
};
template <typename T>
struct ColumnSide<T, kEpiSum> {
  float scale;
};
template <typename T>
struct ColumnSide<T, kEpiScaled> {
  float scale;
};

// Ranges of r for a.i rows where `planned` rows would have had a.splits: as many as the launch has blocks for and the
// workspace room.  (1024 rows of a launch made for 2048 x 32256 x 4096: 239 us, 312 in the two ranges of all rows.)
__device__ __forceinline__ int32_t more_splits(const LinArgs& a, int64_t planned) {
  const uint32_t had = (uint32_t)planned, has = (uint32_t)a.i, high = (uint32_t)a.tile_rows;
  const uint32_t blocks = (uint32_t)a.splits * ((had + high - 1) / high) / ((has + high - 1) / high);
  const uint32_t room = (uint32_t)((uint64_t)a.splits * had / has), most = (uint32_t)a.most_splits;
  uint32_t s = blocks < room ? blocks : room;
  if (s > most) s = most;
  return s > (uint32_t)a.splits ? (int32_t)s : a.splits;
}
// The range of r that a block sums.
template <int EPI>
__device__ __forceinline__ uint32_t range_of(const LinArgs& a) {
  return EPI == kEpiSum ? (uint32_t)a.range : blockIdx.y;
}

// Rows of the logits' gradient further up, of all that a part reads and writes by row.
template <typename T>
__device__ __forceinline__ void move_rows(LinArgs& a, int64_t by) {
  using Mem = typename El<T>::Mem;
  a.prod[0].p = static_cast<const Mem*>(a.prod[0].p) + by * a.prod[0].ldp;
  a.out = static_cast<Mem*>(a.out) + by * a.ldout;
  a.targets += by;
  a.lse += by;
  if (a.lse_low) a.lse_low += by;
  if (a.row_scale) a.row_scale += by;
}

// Products of which only some rows are there (LinArgs::count): sets their number, and says whether there are none.
template <typename T, int EPI>
__device__ __forceinline__ bool without_rows(LinArgs& a) {
  if constexpr (EPI == kEpiXentGrad || EPI == kEpiSum || EPI == kEpiScaled) {
    if (a.count) {
      const int64_t rows = *a.count;
      if (EPI == kEpiScaled) {
        if (rows < a.prod[0].r) a.prod[0].r = rows;
      } else {
        const int64_t planned = a.i;
        int64_t from = a.row_from, end = rows;
        if constexpr (EPI == kEpiXentGrad) {
          if (a.first_count) {
            const int64_t first = *a.first_count;
            if (from == 0) {
              end = first;
            } else {
              move_rows<T>(a, first - from);
              from = first;
            }
          }
        }
        if (end - from < a.i) a.i = end - from;
        if (a.i <= 0) return true;
        if constexpr (EPI == kEpiSum) {
          if (a.splits > 1) a.splits = more_splits(a, planned);
        }
        return false;
      }
    }
  }
  return false;
}
// The products that an epilogue's launches sum, by number.  Where without_rows changes one they are chosen between, not
// indexed, so that the arguments stay where they are passed.
template <int EPI>
constexpr bool kOneProduct = EPI == kEpiXent || EPI == kEpiXentGrad;
template <int EPI>
__device__ __forceinline__ decltype(auto) product_of(const LinArgs& a, int32_t second) {
  if constexpr (kOneProduct<EPI>)
    return (a.prod[0]);
  else if constexpr (EPI == kEpiSum || EPI == kEpiScaled)
    return second ? LinProduct(a.prod[1]) : LinProduct(a.prod[0]);
  else
    return (a.prod[second]);
}

// scale[0] / totals[1]; 0 where no row counts.
__device__ __forceinline__ float total_scale(const LinArgs& a) {
  const float s = a.scale ? *a.scale : 1.f;
  if (!a.totals) return s;
  const float count = a.totals[1];
  return count > 0.f ? s / count : 0.f;
}
// Where eight consecutive columns from j0 on hold the target, or -1.
__device__ __forceinline__ int target_place(const LinArgs& a, int64_t target, int64_t j0) {
  const int64_t at = target - a.col0 - j0;
  return at >= 0 && at < 8 ? (int)at : -1;
}

__device__ __forceinline__ int64_t row_blocks(const LinArgs& a) { return (a.j + kCkptBlock - 1) / kCkptBlock; }

// The loads of out[i][j0 .. j0 + 8); nothing where it is not whole (a checkpoint's rows are: they are padded).
// WHOLE: the caller knows that all eight lie inside, here and below.
template <typename T, int EPI, bool WHOLE = false>
__device__ __forceinline__ void side_load(const LinArgs& a, int64_t i, int64_t j0, Side<T, EPI>& s) {
  using Mem = typename El<T>::Mem;
  if constexpr (EPI == kEpiLayer) {
    if (WHOLE || (i < a.i && j0 + 8 <= a.j)) {
      if (a.mul) s.mul.load(static_cast<const Mem*>(a.mul) + i * a.ldmul + j0);
      if (a.residual) s.residual.load(static_cast<const Mem*>(a.residual) + i * a.ldres + j0);
    }
  }
  if constexpr (EPI == kEpiDgrad) {
    if (a.z_codes && (WHOLE || (i < a.i && j0 < a.j))) {
      const int64_t nb = row_blocks(a), at = i * nb * kCkptBlock + j0, block = i * nb + j0 / kCkptBlock;
      s.z = *reinterpret_cast<const u32x2*>(a.z_codes + at);
      s.z_byte = a.z_exps[block];
      if (a.up_codes) {
        s.up = *reinterpret_cast<const u32x2*>(a.up_codes + at);
        s.up_byte = a.up_exps[block];
      }
    }
  }
  if constexpr (EPI == kEpiXent) {
    if (WHOLE || i < a.i) s.target = a.targets[i];
  }
  if constexpr (EPI == kEpiXentGrad) {
    if (WHOLE || i < a.i) {
      s.target = a.targets[i];
      s.lse = a.lse[i];
      s.low = a.lse_low ? a.lse_low[i] : 0.f;
      s.scale = a.row_scale ? a.row_scale[i] : 1.f;
    }
  }
  if constexpr (EPI == kEpiSum) {
    if (WHOLE || (i < a.i && j0 < a.j)) {
      if (a.sum_in) s.sum.load(a.sum_in + i * a.ldsum + j0);  // rows of whole eights
      s.row = a.out_rows ? a.out_rows[i] : a.targets && a.targets[i] == a.ignore ? -1 - i : i;
    }
  }
}

template <typename T, int EPI>
__device__ __forceinline__ void column_load(const LinArgs& a, int64_t j0, ColumnSide<T, EPI>& s) {
  if constexpr (EPI == kEpiLayer) {
    if (a.bias && j0 + 8 <= a.j) s.bias.load(static_cast<const typename El<T>::Mem*>(a.bias) + j0);
  }
  if constexpr (EPI == kEpiSum || EPI == kEpiScaled) s.scale = total_scale(a);
}

// One side matrix's values: loaded ahead, or at a row's end element by element.
template <typename T>
__device__ __forceinline__ void side_values(const Raw8<T>& raw, const void* row, int64_t j0, int64_t valid, float u[8]) {
  raw.get(u);
  if (valid < 8) {
    const auto* p = static_cast<const typename El<T>::Mem*>(row) + j0;
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = e < valid ? El<T>::load(p + e) : 0.f;
  }
}

// ---------------------------------------------------------------- statistics of logits
// exp(v - top) as the sums take it: by the hardware's exp2 in bf16 (a token's loss is off by up to 4e-7 of itself so).  The difference is taken first: one fused operation with top
// log2 e rounded would be off by its rounding, which passes exp2's range where logits are 2^31.
template <typename T>
struct StatExp {
  float top;
  __device__ __forceinline__ explicit StatExp(float t) : top(t == -__builtin_inff() ? 0.f : t) {}  // only -inf: a sum of zeros
  __device__ __forceinline__ float operator()(float v) const {
    if constexpr (El<T>::kBytes == 4)
      return expf(v - top);
    else
      return __builtin_amdgcn_exp2f((v - top) * 1.44269504088896340736f);
  }
};
// exp(v - lse - low), low being what lse's rounding left: up to 13 where logits are so large, and most often far below 1.
template <typename T>
__device__ __forceinline__ float grad_exp(float v, float lse, float low) {
  if constexpr (El<T>::kBytes == 4)
    return expf((v - lse) - low);
  else
    return __builtin_amdgcn_exp2f(__builtin_fmaf(v - lse, 1.44269504088896340736f, low * -1.44269504088896340736f));
}
// (top, sum) of two sets of values: sum = sum exp(v - top), and exp(v - 0) where there is only -inf.
__device__ __forceinline__ void join_stats(float& top, float& sum, float other_top, float other_sum) {
  const float t = fmaxf(top, other_top), from = t == -__builtin_inff() ? 0.f : t;
  sum = sum * expf(top - from) + other_sum * expf(other_top - from);
  top = t;
}
// Row i's values v[8] of columns j0 on, of which `valid` exist, the rest of the row's tile in the LANES - 1 neighbouring lanes:
// its largest value and sum of exponentials, written by the first lane to stats number `slot`, and its target's logit.
template <typename T, int LANES>
__device__ __forceinline__ void eight_stats(const LinArgs& a, int64_t i, int64_t j0, int64_t valid, const float v[8],
                                            int64_t target, int64_t slot) {
  float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = e < valid ? fmaxf(top, v[e]) : top;
  top = lanes_max<LANES>(top);
  const StatExp<T> from(top);
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += e < valid ? from(v[e]) : 0.f;
  sum = lanes_sum<LANES>(sum);
  if (i >= a.i) return;
  if (valid > 0) {
    const int at = target_place(a, target, j0);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e == at && e < valid) a.target_z[i] = v[e];
  }
  if ((threadIdx.x & (LANES - 1)) == 0) *reinterpret_cast<f32x2*>(a.stats + (i * a.stat_ld + slot) * 2) = f32x2{top, sum};
}

// The epilogue on out[i][j0 .. j0 + 8), j0 a multiple of 8, with what column_load and side_load loaded for it;
// the four lanes of a checkpoint block differ in lane bits A and B.  Every lane of the wave calls it (i or j0 may
// lie outside).
template <typename T, int EPI, int A, int B, bool WHOLE = false>
__device__ __forceinline__ void epilogue8(const LinArgs& a, int64_t i, int64_t j0, float v[8], const ColumnSide<T, EPI>& c,
                                          const Side<T, EPI>& s) {
  using Mem = typename El<T>::Mem;
  const bool row = WHOLE || i < a.i;
  const int64_t valid = WHOLE ? 8 : row ? a.j - j0 : 0;
  if constexpr (EPI == kEpiLayer) {
    float u[8];
    if (a.bias && valid > 0) {
      side_values<T>(c.bias, a.bias, j0, valid, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    if (a.codes) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < valid ? v[e] : 0.f;
      const uint32_t byte = ckpt_byte(block_max<A, B>(v));
      const int64_t nb = row_blocks(a);
      if (WHOLE || (row && j0 < nb * kCkptBlock)) {
        *reinterpret_cast<u32x2*>(a.codes + i * nb * kCkptBlock + j0) = ckpt_pack8(v, byte);
        if (j0 % kCkptBlock == 0) a.exps[i * nb + j0 / kCkptBlock] = (uint8_t)byte;
      }
    }
    if (valid <= 0) return;
    if (a.act != SMAT_ACT_NONE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = act_value<T>(v[e], a.act);
    }
    if (a.mul) {
      side_values<T>(s.mul, static_cast<const Mem*>(a.mul) + i * a.ldmul, j0, valid, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= u[e];
    }
    if (a.residual) {
      side_values<T>(s.residual, static_cast<const Mem*>(a.residual) + i * a.ldres, j0, valid, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
  }
  if (valid <= 0) return;
  if constexpr (EPI == kEpiXentGrad) {  // out's rows hold whole eights: zeros past the last column
    const bool outside = s.target < 0 || s.target >= a.classes;
    const float scale = outside ? __builtin_nanf("") : s.scale;
    if (s.target == a.ignore) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
    } else {
      const int at = target_place(a, s.target, j0);
      float hit = 0.f;
      if (at >= 0) {  // one eight of a row: expm1 keeps what p - 1 would lose where p is nearly 1
#pragma unroll
        for (int e = 0; e < 8; ++e) hit = e == at ? v[e] : hit;
        hit = expm1f((hit - s.lse) - s.low) * scale;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = grad_exp<T>(v[e], s.lse, s.low) * scale;
      if (at >= 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e == at ? hit : v[e];
      }
    }
    if (!WHOLE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < valid ? v[e] : 0.f;
    }
    El<T>::store8(static_cast<Mem*>(a.out) + i * a.ldout + j0, v);
    if constexpr (El<T>::kBytes == 2) {
      if (a.out_low) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] -= bf16_to_f32(to_bf16(v[e]));
        El<T>::store8(static_cast<Mem*>(a.out_low) + i * a.ldout + j0, v);
      }
    }
    return;
  }
  if constexpr (EPI == kEpiSum) {
    if (a.sum_in) {
      float u[8];
      s.sum.get(u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    if (a.sum_out) {
      El<float>::store8(a.sum_out + i * a.ldsum + j0, v);
      return;
    }
  }
  if constexpr (EPI == kEpiSum || EPI == kEpiScaled) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= c.scale;
  }
  if constexpr (EPI == kEpiSum) {
    i = s.row;
    if (i < 0) {
      i = -1 - i;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
  }
  if constexpr (EPI == kEpiDgrad) {
    if (a.z_codes) {
      float z[8];
      ckpt_unpack8(s.z, s.z_byte, z);
      if (a.up_codes) {
        float u[8], w[8];
        ckpt_unpack8(s.up, s.up_byte, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float value, slope;
          act_both<T>(z[e], a.act, value, slope);
          w[e] = v[e] * value;
          v[e] *= slope * u[e];
        }
        store_row8<T>(static_cast<Mem*>(a.out_up) + i * a.ldup + j0, valid, w);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float value, slope;
          act_both<T>(z[e], a.act, value, slope);
          v[e] *= slope;
        }
      }
    }
  }
  store_row8<T>(static_cast<Mem*>(a.out) + i * a.ldout + j0, valid, v);
}

}  // namespace smat
