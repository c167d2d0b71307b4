// Checks of the arguments that the C ABI's calls on matrices share: dimensions, dtypes, row strides, alignment,
// overlap and workspaces.
#pragma once

#include "smat.h"
#include "smat_error.h"
#include "smat_linear.h"

namespace smat {

constexpr int64_t kMaxDim = INT32_MAX;
constexpr int64_t kMaxSpan = 1ll << 60;
constexpr int64_t kMaxGrid = INT32_MAX;

inline size_t dtype_bytes(int d) { return d == SMAT_F32 ? 4 : 2; }

inline smat_status check_types(int dtype, int act, const char* where) {
  if (dtype != SMAT_F32 && dtype != SMAT_BF16) return fail(SMAT_ERR_DTYPE, "%s: unsupported dtype", where);
  if (act < SMAT_ACT_NONE || act > SMAT_ACT_SILU) return fail(SMAT_ERR_INVALID, "%s: unknown activation %d", where, act);
  return SMAT_OK;
}

// One array of a call, as the checks see it: `rows` runs of `run` bytes, `ld` bytes apart.
struct Array {
  const char* what;
  const void* p;
  int64_t rows, run, ld;
  size_t align;
  bool out;
  bool same;  // may be one of the outputs itself

  int64_t span() const { return rows > 0 && run > 0 ? (rows - 1) * ld + run : 0; }
};

// A row stride that check_arrays refuses stays one in bytes.
inline Array matrix(const char* what, const void* p, int64_t rows, int64_t cols, int64_t ld, int dtype, bool out = false,
             bool same = false) {
  const int64_t b = (int64_t)dtype_bytes(dtype);
  const int64_t bytes = ld < 0 ? -1 : ld > kMaxSpan ? INT64_MAX : ld * b;
  return Array{what, p, rows, cols * b, bytes, (size_t)b, out, same};
}
inline Array codes(const char* what, const void* p, int64_t rows, int64_t cols, bool out = false) {
  const int64_t run = ckpt_blocks(cols) * kCkptBlock;
  return Array{what, p, rows, run, run, 16, out, false};
}
inline Array exps(const char* what, const void* p, int64_t rows, int64_t cols, bool out = false) {
  const int64_t run = ckpt_blocks(cols);
  return Array{what, p, rows, run, run, 1, out, false};
}

inline bool overlap(const Array& a, const Array& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  if (!(x < y + (uintptr_t)b.span() && y < x + (uintptr_t)a.span())) return false;
  if (a.ld == b.ld && a.ld > 0) {  // columns of one buffer: disjoint where neither run reaches the other
    const int64_t d = (int64_t)(y > x ? (y - x) % (uintptr_t)a.ld : (a.ld - (int64_t)((x - y) % (uintptr_t)a.ld)) % a.ld);
    if (d >= a.run && d + b.run <= a.ld) return false;
  }
  return true;
}

// Row strides that address every row, element alignment, pointers where there is something to access, and outputs
// apart from everything else.
inline smat_status check_arrays(const Array* arrays, int count, const char* where) {
  for (int i = 0; i < count; ++i) {
    const Array& a = arrays[i];
    if (a.rows == 0 || a.run == 0) continue;
    if (!a.p) return fail(SMAT_ERR_INVALID, "%s: %s is NULL", where, a.what);
    if (a.ld < a.run) return fail(SMAT_ERR_INVALID, "%s: row stride of %s is below its columns", where, a.what);
    if (a.ld > kMaxSpan / a.rows) return fail(SMAT_ERR_INVALID, "%s: %s is too large", where, a.what);
    if (reinterpret_cast<uintptr_t>(a.p) % a.align)
      return fail(SMAT_ERR_INVALID, "%s: %s must be aligned to %zu bytes", where, a.what, a.align);
  }
  for (int i = 0; i < count; ++i)
    for (int j = 0; j < count; ++j) {
      const Array &a = arrays[i], &b = arrays[j];
      if (i == j || !a.out || (b.out && j < i) || a.span() == 0 || b.span() == 0 || !overlap(a, b)) continue;
      if (a.same && b.same && a.p == b.p && a.ld == b.ld) continue;
      return fail(SMAT_ERR_INVALID, "%s: %s overlaps %s", where, a.what, b.what);
    }
  return SMAT_OK;
}

inline smat_status check_dims(const int64_t* dims, int count, const char* where) {
  for (int i = 0; i < count; ++i)
    if (dims[i] < 0 || dims[i] > kMaxDim)
      return fail(SMAT_ERR_INVALID, "%s: dimensions must lie in [0, 2^31 - 1]", where);
  return SMAT_OK;
}

// The launches count blocks of 32 x 8 outputs and tiles in 31 bits.
inline smat_status check_grid(int64_t rows, int64_t cols, const char* where) {
  if (rows > 0 && ckpt_blocks(cols) > kMaxGrid * 64 / rows) return fail(SMAT_ERR_INVALID, "%s: too large", where);
  return SMAT_OK;
}

inline smat_status check_workspace(const void* workspace, size_t have, size_t need, const char* where) {
  if (need == 0) return SMAT_OK;
  if (!workspace || have < need)
    return fail(SMAT_ERR_INVALID, "%s: workspace of %zu bytes, %zu are needed", where, have, need);
  if (reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(SMAT_ERR_INVALID, "%s: workspace must be aligned to 16 bytes", where);
  return SMAT_OK;
}

inline size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace smat
