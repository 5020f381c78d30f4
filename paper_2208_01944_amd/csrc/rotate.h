// Internal interface of the head norms and rotation (k_rotate.hip).
#pragma once

#include "serve_common.h"

namespace palq {

struct RotateArgs {
  BatchView b;
  TreeView tree;
  // queries and keys: values, results, weights (nullable), heads (0: none), strides in elements
  const void *x[2];
  void *y[2];
  const float *w[2];
  int32_t heads[2];
  int64_t x_row[2], x_head[2], y_row[2], y_head[2];
  const uint64_t *phase;  // turns a position, in 2^-64 of one
  int32_t pairs, interleaved, dim;
  float eps;              // 0: no norm
};

hipError_t launch_rotate(const RotateArgs &a, int type, hipStream_t s);

}  // namespace palq
