// The paged 8-bit cache: append (quantise new keys and values into their
// pages) and read (the values that cached codes stand for).
//
// A block is one page of one head, with one scale for its keys and one for its
// values.  Appending n tokens behind the o that the block holds:
//   s = max(s_old (o > 0), max|new| fl(1/127), 2^-100)
//   old codes: rint(code (s_old / s)) where s > s_old; new: rint(x fl(1/s)).
// Keys lie token by token, [page][dim], values channel by channel,
// [dim][page]: each is the order in which the attention's matrix operand takes
// 16 consecutive bytes.
//
// Both directions are bound by memory: a workgroup takes one (request, block,
// head, keys or values), its threads 16 codes at a time.
#include <algorithm>

#include "cache.h"
#include "serve_common.h"

namespace palq {

namespace {

__device__ __forceinline__ int page_of(const CacheView &c, const BatchView &b, int r, int block) {
  if (block >= b.max_pages) return -1;
  const int pid = b.table[(int64_t)r * b.max_pages + block];
  return pid >= 0 && pid < c.pages ? pid : -1;
}

// 16 old codes under a grown scale.
__device__ __forceinline__ v4i rescale16(v4i o, float ratio) {
  v4i out;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float t = (float)(int8_t)((uint32_t)o[q] >> (8 * i)) * ratio;
      w |= ((uint32_t)(int)__builtin_rintf(t) & 0xffu) << (8 * i);
    }
    out[q] = (int)w;
  }
  return out;
}

struct NewKv {
  const void *k, *v;
  int64_t k_row, k_head, v_row, v_head;  // strides in elements; a row's channels are consecutive
};

template <class T>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, BatchView b, NewKv x) {
  typedef typename T::raw R;
  __shared__ uint32_t part[4];
  const int r = blockIdx.z >> 1, h = blockIdx.y;
  const bool values = blockIdx.z & 1;
  const Request q = request_of(b, r, c.shift);
  const int old = max(0, q.len - q.n);  // rows before position 0 have no place
  const int block = (old >> c.shift) + (int)blockIdx.x;
  const int t0 = block << c.shift, lo = max(old, t0), hi = min(q.len, t0 + c.page);
  if (lo >= hi) return;
  const int pid = page_of(c, b, r, block);
  if (pid < 0) return;
  const int kept = lo - t0, n = hi - lo, D = c.dim;
  const R *src = (const R *)(values ? x.v : x.k);
  const int64_t row = values ? x.v_row : x.k_row, head = values ? x.v_head : x.k_head;
  src += (q.row0 + (lo - (q.len - q.n))) * row + h * head;  // row of token lo
  const bool vec = (((uintptr_t)src | (uintptr_t)(row * sizeof(R))) & 15u) == 0;

  // largest magnitude of the new values
  uint32_t mag = 0;
  const int pd = D / 16;
  for (int p = threadIdx.x; p < n * pd; p += 256) {
    float v[16];
    load16<T>(src + (int64_t)(p / pd) * row + p % pd * 16, 16, vec, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) mag = max(mag, mag_bits(v[i]));
  }
  mag = wave_max(mag);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mag;
  const int64_t ph = (int64_t)pid * c.heads + h;
  float *scale = (values ? c.vs : c.ks) + ph;
  const float had = kept ? *scale : 0.0f;
  __syncthreads();
  mag = max(max(part[0], part[1]), max(part[2], part[3]));
  float s = scale_of(mag);
  if (kept && !(s > had)) s = s == s ? had : s;  // (had NaN stays)
  const float inv = inverse_of(s), ratio = had / s;
  const bool bad = !(s == s), grown = kept && !bad && s > had;
  if (threadIdx.x == 0) *scale = s;
  int8_t *dst = (values ? c.v : c.k) + ph * c.page * D;
  if (!values) {
    for (int p = threadIdx.x; p < n * pd; p += 256) {
      float v[16];
      load16<T>(src + (int64_t)(p / pd) * row + p % pd * 16, 16, vec, v);
      *(v4i *)(dst + (int64_t)(kept + p / pd) * D + p % pd * 16) = bad ? v4i{0, 0, 0, 0} : quantize16(v, inv);
    }
    if (grown)
      for (int p = threadIdx.x; p < kept * pd; p += 256) ((v4i *)dst)[p] = rescale16(((const v4i *)dst)[p], ratio);
  } else {
    // a piece: 16 tokens of one channel; neighbouring lanes take neighbouring channels
    const int c0 = grown ? 0 : kept >> 4, pieces = ((hi - t0 + 15) >> 4) - c0;
    for (int p = threadIdx.x; p < pieces * D; p += 256) {
      const int d = p % D, at = (c0 + p / D) * 16;
      v4i *piece = (v4i *)(dst + (int64_t)d * c.page + at);
      v4i o = {0, 0, 0, 0};
      if (at < kept) {
        o = *piece;
        if (grown) o = rescale16(o, ratio);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = at + i - kept;
        if (t >= 0) {
          const int code = t < n && !bad ? code_of(T::get(src[(int64_t)t * row + d]), inv) : 0;
          o[i >> 2] = (int)(((uint32_t)o[i >> 2] & ~(0xffu << (8 * (i & 3)))) | ((uint32_t)code & 0xffu) << (8 * (i & 3)));
        }
      }
      *piece = o;
    }
  }
}

struct OutKv {
  void *k, *v;
  int64_t k_row, k_head, v_row, v_head;
};

template <class T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheView c, BatchView b, OutKv x) {
  typedef typename T::raw R;
  const int r = blockIdx.z >> 1, h = blockIdx.y;
  const bool values = blockIdx.z & 1;
  const Request q = request_of(b, r, c.shift);
  const int first = max(0, q.len - q.n);
  const int block = (first >> c.shift) + (int)blockIdx.x;
  const int t0 = block << c.shift, lo = max(first, t0), hi = min(q.len, t0 + c.page);
  if (lo >= hi) return;
  const int pid = page_of(c, b, r, block), D = c.dim;
  const int64_t ph = (int64_t)max(pid, 0) * c.heads + h;
  const float s = pid < 0 ? 0.0f : (values ? c.vs : c.ks)[ph];
  const int8_t *src = (values ? c.v : c.k) + ph * c.page * D;
  const int64_t row = values ? x.v_row : x.k_row, head = values ? x.v_head : x.k_head;
  R *dst = (R *)(values ? x.v : x.k) + (q.row0 + (lo - (q.len - q.n))) * row + h * head;
  const bool al = (((uintptr_t)dst | (uintptr_t)(row * sizeof(R))) & (4 * sizeof(R) - 1)) == 0;
  if (!values) {
    const int quads = D / 4;
    for (int p = threadIdx.x; p < (hi - lo) * quads; p += 256) {
      const int t = p / quads, d = p % quads * 4;
      const uint32_t w = *(const uint32_t *)(src + (int64_t)(lo - t0 + t) * D + d);
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i)) * s;
      store4<T>(dst + (int64_t)t * row + d, v, al);
    }
  } else {
    const int c0 = (lo - t0) >> 4, pieces = ((hi - t0 + 15) >> 4) - c0;
    for (int p = threadIdx.x; p < pieces * D; p += 256) {
      const int d = p % D, at = (c0 + p / D) * 16;
      const v4i o = *(const v4i *)(src + (int64_t)d * c.page + at);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = t0 + at + i;
        if (t >= lo && t < hi) dst[(int64_t)(t - lo) * row + d] = T::put((float)(int8_t)((uint32_t)o[i >> 2] >> (8 * (i & 3))) * s);
      }
    }
  }
}

// Blocks that max_new tokens behind any number of old ones can touch.
unsigned blocks_of(const CacheView &c, const BatchView &b) {
  const int64_t n = std::min<int64_t>(b.max_new, b.max_len);
  return (unsigned)std::min<int64_t>((n + c.page - 2) / c.page + 1, b.max_pages);
}

}  // namespace

hipError_t launch_cache_append(const CacheView &c, const BatchView &b, const void *k, const void *v, int type,
                               const int64_t *stride, hipStream_t s) {
  const dim3 g(blocks_of(c, b), (unsigned)c.heads, (unsigned)b.requests * 2);
  const NewKv x{k, v, stride[0], stride[1], stride[2], stride[3]};
  if (type == PALQ_F32) cache_append_kernel<F32><<<g, 256, 0, s>>>(c, b, x);
  else if (type == PALQ_F16) cache_append_kernel<F16><<<g, 256, 0, s>>>(c, b, x);
  else cache_append_kernel<BF16><<<g, 256, 0, s>>>(c, b, x);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheView &c, const BatchView &b, void *k, void *v, int type, const int64_t *stride,
                             hipStream_t s) {
  const dim3 g(blocks_of(c, b), (unsigned)c.heads, (unsigned)b.requests * 2);
  const OutKv x{k, v, stride[0], stride[1], stride[2], stride[3]};
  if (type == PALQ_F32) cache_read_kernel<F32><<<g, 256, 0, s>>>(c, b, x);
  else if (type == PALQ_F16) cache_read_kernel<F16><<<g, 256, 0, s>>>(c, b, x);
  else cache_read_kernel<BF16><<<g, 256, 0, s>>>(c, b, x);
  return hipGetLastError();
}

}  // namespace palq
