// Internal launcher of rope.hip; arguments are checked in abi_rope.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace losa {

// Rotary positions and query/key norms (rope.hip).  One tensor's share of a call:
// [B][N][H][d] rows at x, strides in elements, to [B][n_pad][H] rows at y.
constexpr int kMaxAxes = 4;
constexpr int kNormNone = 0, kNormRms = 1, kNormLayer = 2;
struct RowsTensor {
  const void* x;
  void* y;
  const float* w;  // weight and bias of the norm, or null
  const float* b;
  int64_t xb, xt, xh, yb, yt, yh;
  int H, norm, rotate;
  int hc, chunks;  // heads per wave and their number (set by the launcher)
};
struct RowsArgs {
  RowsTensor t[3];
  int64_t blocks[3];  // workgroups of each tensor (set by the launcher)
  int B, N, n_pad, tiles;
  float eps;
  const float* table;
  const int32_t* pos;  // [batches][axes][N]
  int64_t pos_batch;
  int axes, rot8;  // rotated dims / 8
  int pair0[kMaxAxes], dim[kMaxAxes], len[kMaxAxes], off[kMaxAxes];  // by axis
};
// all: one norm over the H rows of a token (every tensor of the call that has a norm)
hipError_t launch_rows(int d, bool bf16, bool halves, RowsArgs& a, int tensors, bool all,
                       hipStream_t stream);

}  // namespace losa
