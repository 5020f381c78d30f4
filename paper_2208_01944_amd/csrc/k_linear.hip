// Matrix product in 8-bit integers with a scale for each token and channel:
//   y[m][n] = (sum_k x[m][k] w[n][k]) s[m] t[n] + b[n]
// x codes formed from floating values within the call (one scale a token) or
// given; w codes laid out once.  The sum is exact in int32 (k < 2^17).
//
// Operand order.  Both matrices are kept as slabs of 16 rows x 64 k, 1 KB:
// 16-byte piece (k / 16 % 4) * 16 + (row % 16) holds 16 consecutive k of a row,
// which is lane for lane the operand of v_mfma_i32_16x16x64_i8, and two slabs
// of neighbouring rows are the two operands of v_mfma_i32_32x32x32_i8.  Slabs
// follow each other along k, then along rows.  k is padded to whole blocks
// with zero codes, rows to whole tiles with rows whose results are not stored.
#include <algorithm>

#include "linear.h"
#include "serve_common.h"

namespace palq {

namespace {

// ------------------------------------------------------------ token quantiser
// WPR waves a row; SLABS: codes into slabs, else row by row.  A lane takes 16
// consecutive columns at a time and keeps the first kHeld such pieces in
// registers between the two looks at a row (largest magnitude, then codes).
constexpr int kHeld = 4;

template <class T, int WPR, bool SLABS>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const typename T::raw *x, int64_t rows, int cols, int64_t ld,
                                                            int kp, int8_t *codes, int64_t codes_ld, float *scales) {
  constexpr int RB = 4 / WPR, LANES = 64 * WPR;
  __shared__ uint32_t part[4];
  const int wave = threadIdx.x >> 6, lr = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * RB + (WPR == 1 ? wave : 0);
  const bool live = row < rows;
  const typename T::raw *xr = x + (live ? row : 0) * ld;
  const bool vec = (((uintptr_t)x | (uintptr_t)(ld * sizeof(typename T::raw))) & 15u) == 0;
  float held[kHeld][16];
  uint32_t mag = 0;
  const int pieces = live ? kp / 16 : 0;
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const int p = h * LANES + lr;
    if (p < pieces) load16<T>(xr + p * 16, cols - p * 16, vec, held[h]);
  }
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (h * LANES + lr < pieces)
#pragma unroll
      for (int i = 0; i < 16; ++i) mag = max(mag, mag_bits(held[h][i]));
  for (int p = kHeld * LANES + lr; p < pieces; p += LANES) {
    float v[16];
    load16<T>(xr + p * 16, cols - p * 16, vec, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) mag = max(mag, mag_bits(v[i]));
  }
  mag = wave_max(mag);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) part[wave] = mag;
    __syncthreads();
    mag = max(max(part[0], part[1]), max(part[2], part[3]));
  }
  if (!live) return;
  const float s = scale_of(mag), inv = inverse_of(s);
  const bool bad = !(s == s);
  if (lr == 0) scales[row] = s;
  const bool out16 = !SLABS && (((uintptr_t)codes | (uintptr_t)codes_ld) & 15u) == 0;
  auto put = [&](int p, const float *v) __attribute__((always_inline)) {
    const v4i o = bad ? v4i{0, 0, 0, 0} : quantize16(v, inv);
    if constexpr (SLABS) {
      const int64_t at = ((row >> 4) * (kp / 64) + (p >> 2)) * 1024 + (p & 3) * 256 + (row & 15) * 16;
      *(v4i *)(codes + at) = o;
    } else {
      int8_t *dst = codes + row * codes_ld + p * 16;
      const int n = cols - p * 16;
      if (out16 && n >= 16) {
        *(v4i *)dst = o;
      } else {
        for (int i = 0; i < 16; ++i)
          if (i < n) dst[i] = (int8_t)((uint32_t)o[i >> 2] >> (8 * (i & 3)));
      }
    }
  };
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (h * LANES + lr < pieces) put(h * LANES + lr, held[h]);
  for (int p = kHeld * LANES + lr; p < pieces; p += LANES) {
    float v[16];
    load16<T>(xr + p * 16, cols - p * 16, vec, v);
    put(p, v);
  }
}

// Codes in rows (weights, or activations given as codes) into slabs: a thread a
// piece, so a wave reads 64 bytes of 16 rows and writes a whole slab.
__global__ __launch_bounds__(256) void slab_kernel(const int8_t *x, int64_t rows, int64_t slab_rows, int cols, int64_t ld,
                                                   int kp, int8_t *out) {
  const int64_t slab = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int per = kp / 64;
  const int64_t rt = slab / per;
  if (rt >= slab_rows) return;
  const int lane = threadIdx.x & 63;
  const int64_t row = rt * 16 + (lane & 15);
  const int k = (int)(slab - rt * per) * 64 + (lane >> 4) * 16;
  v4i o = {0, 0, 0, 0};
  if (row < rows && k < cols) {
    const int8_t *p = x + row * ld + k;
    if (k + 16 <= cols && (((uintptr_t)x | (uintptr_t)ld) & 15u) == 0) {
      o = *(const v4i *)p;
    } else {
      for (int i = 0; i < 16; ++i)
        if (k + i < cols) o[i >> 2] |= (int)((uint32_t)(uint8_t)p[i] << (8 * (i & 3)));
    }
  }
  *(v4i *)(out + slab * 1024 + lane * 16) = o;
}

// ------------------------------------------------------------ few tokens
// A workgroup of 4 waves takes 16 channels x 16 MT tokens; each wave a quarter
// of k, operands straight from memory into registers; the waves' sums meet in
// LDS (integers: any order gives the same sum).
template <class T, int MT>
__global__ __launch_bounds__(256) void linear_few_kernel(LinearArgs a) {
  __shared__ v4i part[4][MT][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t nt = blockIdx.x, mt0 = (int64_t)blockIdx.y * MT;
  const int kb = a.kp / 64;
  const v4i *w = (const v4i *)(a.w + nt * kb * 1024) + lane;
  const v4i *x = (const v4i *)(a.x + mt0 * kb * 1024) + lane;
  v4i acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = v4i{0, 0, 0, 0};
#pragma unroll 4
  for (int k = wave; k < kb; k += 4) {
    const v4i wv = w[(int64_t)k * 64];
#pragma unroll
    for (int m = 0; m < MT; ++m)
      acc[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, x[((int64_t)m * kb + k) * 64], acc[m], 0, 0, 0);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) part[wave][m][lane] = acc[m];
  __syncthreads();
  // lane: token lane % 16, channels (lane / 16) * 4 ..
  const bool y4 = (((uintptr_t)a.y | (uintptr_t)(a.y_ld * sizeof(typename T::raw))) & (4 * sizeof(typename T::raw) - 1)) == 0;
  for (int m = wave; m < MT; m += 4) {
    const v4i s = part[0][m][lane] + part[1][m][lane] + part[2][m][lane] + part[3][m][lane];
    const int64_t row = (mt0 + m) * 16 + (lane & 15);
    const int n = (int)nt * 16 + (lane >> 4) * 4;
    if (row >= a.rows || n >= a.n_out) continue;
    const float sc = a.x_scale[row];
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = min(n + i, a.n_out - 1);
      v[i] = (float)s[i] * sc * a.w_scale[c];
      if (a.bias) v[i] += a.bias[c];
    }
    typename T::raw *y = (typename T::raw *)a.y + row * a.y_ld + n;
    if (n + 4 <= a.n_out) {
      store4<T>(y, v, y4);
    } else {
      for (int i = 0; i < 4; ++i)
        if (n + i < a.n_out) y[i] = T::put(v[i]);
    }
  }
}

template <class T>
hipError_t launch_linear_t(const LinearArgs &a, hipStream_t s) {
  const unsigned nt = (unsigned)((a.n_out + 15) / 16);
  const int64_t mt = (a.rows + 15) / 16;
  if (mt <= 1) linear_few_kernel<T, 1><<<dim3(nt, 1), 256, 0, s>>>(a);
  else if (mt <= 2) linear_few_kernel<T, 2><<<dim3(nt, 1), 256, 0, s>>>(a);
  else linear_few_kernel<T, 4><<<dim3(nt, (unsigned)((mt + 3) / 4)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <class T>
void launch_quantize_t(const void *x, int64_t rows, int cols, int64_t ld, int kp, int8_t *codes, int64_t codes_ld,
                       bool slabs, float *scales, hipStream_t s) {
  typedef typename T::raw R;
  // 4 waves a row while that leaves CUs without work
  if (rows <= 512) {
    if (slabs) quantize_rows_kernel<T, 4, true><<<(unsigned)rows, 256, 0, s>>>((const R *)x, rows, cols, ld, kp, codes, codes_ld, scales);
    else quantize_rows_kernel<T, 4, false><<<(unsigned)rows, 256, 0, s>>>((const R *)x, rows, cols, ld, kp, codes, codes_ld, scales);
  } else {
    const unsigned g = (unsigned)((rows + 3) / 4);
    if (slabs) quantize_rows_kernel<T, 1, true><<<g, 256, 0, s>>>((const R *)x, rows, cols, ld, kp, codes, codes_ld, scales);
    else quantize_rows_kernel<T, 1, false><<<g, 256, 0, s>>>((const R *)x, rows, cols, ld, kp, codes, codes_ld, scales);
  }
}

}  // namespace

hipError_t launch_quantize_rows(const void *x, int type, int64_t rows, int cols, int64_t ld, int kp, int8_t *codes,
                                int64_t codes_ld, bool slabs, float *scales, hipStream_t s) {
  if (type == PALQ_F32) launch_quantize_t<F32>(x, rows, cols, ld, kp, codes, codes_ld, slabs, scales, s);
  else if (type == PALQ_F16) launch_quantize_t<F16>(x, rows, cols, ld, kp, codes, codes_ld, slabs, scales, s);
  else launch_quantize_t<BF16>(x, rows, cols, ld, kp, codes, codes_ld, slabs, scales, s);
  return hipGetLastError();
}

hipError_t launch_slabs(const int8_t *x, int64_t rows, int64_t padded_rows, int cols, int64_t ld, int kp, int8_t *out,
                        hipStream_t s) {
  const int64_t slabs = padded_rows / 16 * (kp / 64);
  slab_kernel<<<(unsigned)((slabs + 3) / 4), 256, 0, s>>>(x, rows, padded_rows / 16, cols, ld, kp, out);
  return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &a, int y_type, hipStream_t s) {
  if (y_type == PALQ_F32) return launch_linear_t<F32>(a, s);
  if (y_type == PALQ_F16) return launch_linear_t<F16>(a, s);
  return launch_linear_t<BF16>(a, s);
}

const char *linear_kernel_label(int64_t rows, int n_in, int n_out) { return "linear_few_kernel"; }

}  // namespace palq
