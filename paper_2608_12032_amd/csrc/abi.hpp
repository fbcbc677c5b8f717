// What the files behind include/losa.h share: status reporting and argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include "losa.h"

namespace losa {

// Sets the thread's error text and returns s.
losa_status fail(losa_status s, const char* fmt, ...);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline losa_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return LOSA_OK;
  return fail(LOSA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline size_t elem_bytes(losa_dtype dt) { return dt == LOSA_DTYPE_BF16 ? 2 : 4; }

// Takes a view of [B][N][H] rows of d elements of `el` bytes: *to is `from` with the
// strides that are never used, those along one element, set to d.  Fails on what the
// kernels cannot address, and on an output whose rows overlap along one axis.
losa_status take_view(const char* name, const losa_view* from, losa_view* to, int el, int B,
                      int64_t N, int H, int d, bool out);
// Whether two views that were taken so are the same rows.
bool same_rows(const losa_view& a, const losa_view& b);

}  // namespace losa
