// Internal interface of the 8-bit matrix product (k_linear.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace palq {

constexpr int kLinearK = 128;     // k is padded to a multiple of this
constexpr int kLinearRows = 256;  // rows of either matrix are allocated in multiples of this

struct LinearArgs {
  const int8_t *x, *w;              // slabs
  const float *x_scale, *w_scale;   // per token, per channel
  const float *bias;                // nullable
  void *y;
  int64_t rows, y_ld;
  int32_t n_out, kp;                // kp: padded k
};

// codes: slabs of padded rows (codes_ld unused), or rows of codes_ld bytes with
// kp = cols rounded up to 16.
hipError_t launch_quantize_rows(const void *x, int type, int64_t rows, int cols, int64_t ld, int kp, int8_t *codes,
                                int64_t codes_ld, bool slabs, float *scales, hipStream_t s);
hipError_t launch_slabs(const int8_t *x, int64_t rows, int64_t padded_rows, int cols, int64_t ld, int kp, int8_t *out,
                        hipStream_t s);
hipError_t launch_linear(const LinearArgs &a, int y_type, hipStream_t s);
// Whether a product of floating rows (one row) runs as one launch from them, without slabs of x.
bool linear_one(int64_t rows, int32_t kp);
hipError_t launch_linear_one(const LinearArgs &a, const void *x, int x_type, int32_t n_in, int y_type, hipStream_t s);
// Of floating rows (codes never run as linear_one).
const char *linear_kernel_label(int64_t rows, int n_out, int kp);

}  // namespace palq
