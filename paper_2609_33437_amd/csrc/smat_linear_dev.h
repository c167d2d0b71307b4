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
}

template <typename T, int EPI>
__device__ __forceinline__ void column_load(const LinArgs& a, int64_t j0, ColumnSide<T, EPI>& s) {
  if constexpr (EPI == kEpiLayer) {
    if (a.bias && j0 + 8 <= a.j) s.bias.load(static_cast<const typename El<T>::Mem*>(a.bias) + j0);
  }
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
