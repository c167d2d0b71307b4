// The status and message that an entry point leaves behind (smat_last_error), shared by the files
// that implement the C ABI.
#pragma once

#include "smat.h"

namespace smat {

// Records a printf-style message for smat_last_error() in this thread and returns `st`.
smat_status fail(smat_status st, const char* fmt, ...);

}  // namespace smat

#define SMAT_HIP(call)                                                                         \
  do {                                                                                         \
    hipError_t e_ = (call);                                                                    \
    if (e_ != hipSuccess) return smat::fail(SMAT_ERR_HIP, "%s: %s", #call, hipGetErrorString(e_)); \
  } while (0)
