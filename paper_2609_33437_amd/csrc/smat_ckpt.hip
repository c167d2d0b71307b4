// Activation checkpoints in 8 bits for gfx950: a matrix as int8 multiples of one power of two per 32
// elements of a row, and back (the format is beside ckpt_byte in smat_linear_dev.h).
//
// Both passes are bound by HBM: per element a write moves b + 1 + 1/32 bytes (b = 2 or 4), a read the
// same the other way, plus 1 + 1/32 with a second checkpoint.  A thread holds eight consecutive elements,
// so four neighbouring lanes hold a block and find its maximum with two lane exchanges.
#include "smat_linear_dev.h"

namespace smat {

constexpr int kCkptThreads = 256;

template <typename T>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_write(const typename El<T>::Mem* __restrict__ x, int64_t ld,
                                                             int64_t cols, int64_t nb, int64_t total,
                                                             int8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  // total = rows * nb * 4 eights; a wave's last lanes past it belong to whole blocks of four
  const int64_t t = (int64_t)blockIdx.x * kCkptThreads + threadIdx.x;
  if (t >= total) return;
  const int64_t row = t / (nb * 4), j0 = (t - row * nb * 4) * 8;
  float v[8];
  load_row8<T>(x + row * ld + j0, cols - j0, v);
  const uint32_t byte = ckpt_byte(block_max<1, 2>(v));
  *reinterpret_cast<u32x2*>(codes + t * 8) = ckpt_pack8(v, byte);
  if (t % 4 == 0) exps[t / 4] = (uint8_t)byte;
}

template <typename T>
__global__ __launch_bounds__(kCkptThreads) void k_ckpt_read(const int8_t* __restrict__ codes,
                                                            const uint8_t* __restrict__ exps,
                                                            const int8_t* __restrict__ up_codes,
                                                            const uint8_t* __restrict__ up_exps, int act, int64_t cols,
                                                            int64_t nb, int64_t total,
                                                            typename El<T>::Mem* __restrict__ out, int64_t ldout) {
  const int64_t t = (int64_t)blockIdx.x * kCkptThreads + threadIdx.x;
  if (t >= total) return;
  const int64_t row = t / (nb * 4), j0 = (t - row * nb * 4) * 8;
  float v[8];
  ckpt_unpack8(*reinterpret_cast<const u32x2*>(codes + t * 8), exps[t / 4], v);
  if (act != SMAT_ACT_NONE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<T>(v[e], act);
  }
  if (up_codes) {
    float u[8];
    ckpt_unpack8(*reinterpret_cast<const u32x2*>(up_codes + t * 8), up_exps[t / 4], u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= u[e];
  }
  store_row8<T>(out + row * ldout + j0, cols - j0, v);
}

namespace {
template <typename F>
void with_element(int dtype, F&& fn) {
  if (dtype == 1)
    fn(Bf16());
  else
    fn(float());
}
dim3 ckpt_grid(int64_t total) { return dim3((uint32_t)((total + kCkptThreads - 1) / kCkptThreads)); }
}  // namespace

hipError_t launch_ckpt_write(const void* x, int64_t ld, int64_t rows, int64_t cols, int dtype, int8_t* codes,
                             uint8_t* exps, hipStream_t stream) {
  const int64_t nb = ckpt_blocks(cols), total = rows * nb * 4;
  with_element(dtype, [&](auto tag) {
    using T = decltype(tag);
    k_ckpt_write<T><<<ckpt_grid(total), dim3(kCkptThreads), 0, stream>>>(
        static_cast<const typename El<T>::Mem*>(x), ld, cols, nb, total, codes, exps);
  });
  return hipGetLastError();
}

hipError_t launch_ckpt_read(const int8_t* codes, const uint8_t* exps, const int8_t* up_codes, const uint8_t* up_exps,
                            int act, int64_t rows, int64_t cols, int dtype, void* out, int64_t ldout,
                            hipStream_t stream) {
  const int64_t nb = ckpt_blocks(cols), total = rows * nb * 4;
  with_element(dtype, [&](auto tag) {
    using T = decltype(tag);
    k_ckpt_read<T><<<ckpt_grid(total), dim3(kCkptThreads), 0, stream>>>(
        codes, exps, up_codes, up_exps, act, cols, nb, total, static_cast<typename El<T>::Mem*>(out), ldout);
  });
  return hipGetLastError();
}

}  // namespace smat
