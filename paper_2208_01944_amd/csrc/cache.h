// Internal interface of the paged 8-bit cache and its attention (k_cache.hip,
// k_attend.hip).
#pragma once

#include "serve_common.h"

namespace palq {

// stride: {k row, k head, v row, v head} in elements.
hipError_t launch_cache_append(const CacheView &c, const BatchView &b, const void *k, const void *v, int type,
                               const int64_t *stride, hipStream_t s);
hipError_t launch_cache_read(const CacheView &c, const BatchView &b, void *k, void *v, int type, const int64_t *stride,
                             hipStream_t s);

struct AttendArgs {
  CacheView c;
  BatchView b;
  const uint16_t *q;
  uint16_t *out;
  int64_t q_row, q_head, out_row, out_head;  // strides in elements
  int32_t group;                             // query heads of a cache head
  int32_t causal, window;
  float scale;                               // of the scores
  int32_t block;                             // rows of a workgroup
  int32_t splits;                            // parts that a request's tokens are cut into
  float *part;                               // their results (attend_work_bytes)
};

// Chooses kernel and parts (false: a row tile of all requests is no launch), and the device memory for the parts.
bool attend_plan(AttendArgs &a, int cus);
size_t attend_work_bytes(const AttendArgs &a);
hipError_t launch_attend(const AttendArgs &a, int type, hipStream_t s);

}  // namespace palq
