// Activation checkpoints in 8 bits for gfx950: a matrix as int8 multiples of one power of two per 32
// elements of a row, and back (the format is beside ckpt_byte in smat_linear_dev.h).
//
// Both passes are bound by HBM: per element a write moves b + 1 + 1/32 bytes (b = 2 or 4), a read the
// same the other way, plus 1 + 1/32 with a second checkpoint.  A thread holds eight consecutive elements,
// so four neighbouring lanes hold a block and find its maximum with two lane exchanges.  16384 x 14336 bf16: the write
// takes 115 us, 6.2 TB/s, the read 122 us, 5.8 TB/s, the read with SiLU and a second checkpoint 160 us, 6.0 TB/s;
// 1999 x 4095 fp32, off 16-byte rows, 7.4 us and 9.9 us.
#include <type_traits>

#include "smat_linear_dev.h"

namespace smat {

constexpr int kCkptThreads = 256;

// Where eight number t of the rows lies: FLAT (rows of whole blocks, packed end to end) needs no division.
template <bool FLAT, typename Index>
__device__ __forceinline__ void eight_place(Index t, Index across, int64_t ld, int64_t cols, int64_t& at, int64_t& valid) {
  if constexpr (FLAT) {
    at = (int64_t)t * 8;
    valid = 8;
  } else {
    const Index row = t / across, j0 = (t - row * across) * 8;
    at = (int64_t)row * ld + j0;
    valid = cols - (int64_t)j0;
  }
}

// total = rows * across eights, across = 4 * blocks; a wave's last lanes past it belong to whole blocks of four.
template <typename T, bool FLAT, typename Index>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_write(const typename El<T>::Mem* __restrict__ x, int64_t ld,
                                                             int64_t cols, Index across, int64_t total,
                                                             int8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  const int64_t t = wide_block() * kCkptThreads + threadIdx.x;
  if (t >= total) return;
  int64_t at, valid;
  eight_place<FLAT, Index>((Index)t, across, ld, cols, at, valid);
  float v[8];
  if constexpr (FLAT)
    El<T>::load8(x + at, v);
  else
    load_row8<T>(x + at, valid, v);
  const uint32_t byte = ckpt_byte(block_max<1, 2>(v));
  *reinterpret_cast<u32x2*>(codes + t * 8) = ckpt_pack8(v, byte);
  if (t % 4 == 0) exps[t / 4] = (uint8_t)byte;
}

template <typename T, bool FLAT, typename Index>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_read(const int8_t* __restrict__ codes,
                                                            const uint8_t* __restrict__ exps,
                                                            const int8_t* __restrict__ up_codes,
                                                            const uint8_t* __restrict__ up_exps, int act, int64_t cols,
                                                            Index across, int64_t total,
                                                            typename El<T>::Mem* __restrict__ out, int64_t ldout) {
  const int64_t t = wide_block() * kCkptThreads + threadIdx.x;
  if (t >= total) return;
  const u32x2 z = *reinterpret_cast<const u32x2*>(codes + t * 8);
  const uint32_t z_byte = exps[t / 4];
  u32x2 up = {0u, 0u};
  uint32_t up_byte = 0u;
  if (up_codes) {
    up = *reinterpret_cast<const u32x2*>(up_codes + t * 8);
    up_byte = up_exps[t / 4];
  }
  float v[8];
  ckpt_unpack8(z, z_byte, v);
  if (act != SMAT_ACT_NONE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<T>(v[e], act);
  }
  if (up_codes) {
    float u[8];
    ckpt_unpack8(up, up_byte, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= u[e];
  }
  int64_t at, valid;
  eight_place<FLAT, Index>((Index)t, across, ldout, cols, at, valid);
  if constexpr (FLAT)
    El<T>::store8(out + at, v);
  else
    store_row8<T>(out + at, valid, v);
}

namespace {
template <typename F>
void with_element(int dtype, F&& fn) {
  if (dtype == 1)
    fn(Bf16());
  else
    fn(float());
}
dim3 ckpt_grid(int64_t total) { return wide_grid((total + kCkptThreads - 1) / kCkptThreads); }

// fn(element type, whether the rows are whole blocks end to end, type of an eight's number) of a call.
template <typename F>
void with_place(int dtype, int64_t rows, int64_t cols, int64_t ld, int64_t total, F&& fn) {
  with_element(dtype, [&](auto tag) {
    if (cols % kCkptBlock == 0 && (ld == cols || rows == 1))
      fn(tag, std::true_type(), int64_t());
    else if (total <= INT64_C(0x7FFFFFFF))
      fn(tag, std::false_type(), uint32_t());
    else
      fn(tag, std::false_type(), int64_t());
  });
}
}  // namespace

hipError_t launch_ckpt_write(const void* x, int64_t ld, int64_t rows, int64_t cols, int dtype, int8_t* codes,
                             uint8_t* exps, hipStream_t stream) {
  const int64_t across = ckpt_blocks(cols) * 4, total = rows * across;
  with_place(dtype, rows, cols, ld, total, [&](auto tag, auto flat, auto index) {
    using T = decltype(tag);
    using Index = decltype(index);
    k_ckpt_write<T, flat(), Index><<<ckpt_grid(total), dim3(kCkptThreads), 0, stream>>>(
        static_cast<const typename El<T>::Mem*>(x), ld, cols, (Index)across, total, codes, exps);
  });
  return hipGetLastError();
}

hipError_t launch_ckpt_read(const int8_t* codes, const uint8_t* exps, const int8_t* up_codes, const uint8_t* up_exps,
                            int act, int64_t rows, int64_t cols, int dtype, void* out, int64_t ldout,
                            hipStream_t stream) {
  const int64_t across = ckpt_blocks(cols) * 4, total = rows * across;
  with_place(dtype, rows, cols, ldout, total, [&](auto tag, auto flat, auto index) {
    using T = decltype(tag);
    using Index = decltype(index);
    k_ckpt_read<T, flat(), Index><<<ckpt_grid(total), dim3(kCkptThreads), 0, stream>>>(
        codes, exps, up_codes, up_exps, act, cols, (Index)across, total, static_cast<typename El<T>::Mem*>(out), ldout);
  });
  return hipGetLastError();
}

}  // namespace smat
