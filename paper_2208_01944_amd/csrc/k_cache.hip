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
// head, keys or values).  8 prompts of 113 to 2048 tokens, 8 heads of 128, bf16: append 20
// us (53 MB, 2.6 TB/s), read back as fp32 18 us (89 MB, 4.9 TB/s); 64 single tokens 6 us
// and, their blocks read back, 10: four loads that wait for each other (lengths, table, scale,
// values).
#include <algorithm>

#include "cache.h"
#include "cache_index.h"
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

// A thread's item: 4 tokens x 8 channels, neighbouring lanes neighbouring channels;
// NI items a thread hold a whole block in registers, so new values are read once.
// Values are turned (a word of 4 tokens for each channel) through LDS.
template <class T, int NI>
__global__ __launch_bounds__(kAppendThreads) void cache_append_kernel(CacheView c, BatchView b, NewKv x, int block0) {
  typedef typename T::raw R;
  __shared__ uint32_t part[4];
  __shared__ uint32_t turned[turned_words(NI)];  // [dim][turned_stride]
  const int r = blockIdx.z >> 1, h = blockIdx.y;
  const bool values = blockIdx.z & 1;
  const Request q = request_of(b, r);
  const int old = max(0, q.pos), stop = min(q.len, q.pos + q.n);  // rows before position 0 have no place
  const int block = (old >> c.shift) + block0 + (int)blockIdx.x;
  if (old >= stop || block > (stop - 1) >> c.shift) return;
  const int t0 = block << c.shift, lo = max(old, t0), hi = min(stop, t0 + c.page);
  const int pid = page_of(c, b, r, block);
  if (pid < 0) return;
  const int kept = lo - t0, end = hi - t0, D = c.dim, groups = D / 8, items = append_items(c.page, D);
  const R *src = (const R *)(values ? x.v : x.k);
  const int64_t row = values ? x.v_row : x.k_row, head = values ? x.v_head : x.k_head;
  src += (q.row0 + (t0 - q.pos)) * row + h * head;  // row of token t0 (there may be none)
  const int64_t ph = (int64_t)pid * c.heads + h;
  float *scale = (values ? c.vs : c.ks) + ph;
  const float had = kept ? *scale : 0.0f;

  float v[NI][4][8];
  uint32_t mag = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int p = threadIdx.x + i * kAppendThreads, tq = p / groups * 4, ch = p % groups * 8;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool here = p < items && tq + t >= kept && tq + t < end;
      const R *from = src + (int64_t)(tq + t) * row + ch;
      if (here) {
        load8<T>(from, v[i][t]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][t][j] = 0.0f;
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 8; ++j) mag = max(mag, mag_bits(v[i][t][j]));
  }
  mag = wave_max(mag);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mag;
  __syncthreads();
  mag = max(max(part[0], part[1]), max(part[2], part[3]));
  float s = scale_of(mag);
  if (kept && !(s > had)) s = s == s ? had : s;  // (had NaN stays)
  const float inv = inverse_of(s), ratio = had / s;
  const bool bad = !(s == s), grown = kept && !bad && s > had;
  if (threadIdx.x == 0) *scale = s;
  int8_t *dst = (values ? c.v : c.k) + ph * c.page * D;
  const int words = turned_stride(c.page);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int p = threadIdx.x + i * kAppendThreads, tq = p / groups * 4, ch = p % groups * 8;
    if (p >= items || tq + 4 <= kept || tq >= end) continue;
    uint32_t w[4][2];  // codes of a token's 8 channels
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        w[t][q] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][q] |= bad ? 0u : ((uint32_t)code_of(v[i][t][4 * q + j], inv) & 0xffu) << (8 * j);
      }
    if (!values) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (tq + t >= kept && tq + t < end) *(v2i *)(dst + (tq + t) * D + ch) = v2i{(int)w[t][0], (int)w[t][1]};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // byte j of four tokens
        const int q = j >> 2, at = 8 * (j & 3);
        turned[(ch + j) * words + tq / 4] = (w[0][q] >> at & 0xffu) | (w[1][q] >> at & 0xffu) << 8 | (w[2][q] >> at & 0xffu) << 16 |
                                            (w[3][q] >> at & 0xffu) << 24;
      }
    }
  }
  if (!values) {
    if (grown)
      for (int p = threadIdx.x; p < kept * (D / 16); p += kAppendThreads) ((v4i *)dst)[p] = rescale16(((const v4i *)dst)[p], ratio);
    return;
  }
  __syncthreads();
  // a piece: 16 tokens of one channel; where old ones are among them, or all are and the
  // scale grew, what is there comes first
  const int c0 = grown ? 0 : kept >> 4, pieces = ((end + 15) >> 4) - c0;
  for (int p = threadIdx.x; p < pieces * D; p += kAppendThreads) {
    const int d = p / pieces, at = (c0 + p % pieces) * 16;
    int8_t *to = dst + d * c.page;
    if (at < kept && !grown) {  // only what is new: the old codes need not come first
      for (int t = kept; t < min(end, at + 16); ++t) to[t] = (int8_t)(turned[d * words + (t >> 2)] >> (8 * (t & 3)));
      continue;
    }
    v4i *piece = (v4i *)(to + at);
    v4i o = {0, 0, 0, 0};
    if (at < kept) o = rescale16(*piece, ratio);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = at + 4 * j;
      if (t + 4 <= kept || t >= end) continue;
      const uint32_t fresh = t >= kept ? 0xffffffffu : 0xffffffffu << (8 * (kept - t));
      o[j] = (int)(((uint32_t)o[j] & ~fresh) | (turned[d * words + (t >> 2)] & fresh));
    }
    *piece = o;
  }
}

struct OutKv {
  void *k, *v;
  int64_t k_row, k_head, v_row, v_head;
};

template <class T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheView c, BatchView b, OutKv x, int block0) {
  typedef typename T::raw R;
  const int r = blockIdx.z >> 1, h = blockIdx.y;
  const bool values = blockIdx.z & 1;
  const Request q = request_of(b, r);
  const int first = max(0, q.pos), stop = min(q.len, q.pos + q.n);
  const int block = (first >> c.shift) + block0 + (int)blockIdx.x;
  if (first >= stop || block > (stop - 1) >> c.shift) return;
  const int t0 = block << c.shift, lo = max(first, t0), hi = min(stop, t0 + c.page);
  const int from0 = lo - t0, end = hi - t0;  // the block's tokens that are read
  const int pid = page_of(c, b, r, block), D = c.dim;
  const int64_t ph = (int64_t)max(pid, 0) * c.heads + h;
  const float s = pid < 0 ? 0.0f : (values ? c.vs : c.ks)[ph];
  const int8_t *src = (values ? c.v : c.k) + ph * c.page * D;
  const int64_t row = values ? x.v_row : x.k_row, head = values ? x.v_head : x.k_head;
  R *dst = (R *)(values ? x.v : x.k) + (q.row0 + (lo - q.pos)) * row + h * head;
  // several pieces' loads in flight before the first store
  if (!values) {
    const int quads = D / 4, all = (end - from0) * quads;
    const uint32_t *from = (const uint32_t *)(src + from0 * D);
    for (int p0 = threadIdx.x; p0 < all; p0 += 256 * 8) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = from[min(p0 + i * 256, all - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int p = p0 + i * 256, t = p / quads, d = p % quads * 4;
        if (p >= all) break;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)(int8_t)(w[i] >> (8 * j)) * s;
        store4<T>(dst + (int64_t)t * row + d, v);
      }
    }
  } else {
    const int c0 = from0 >> 4, all = (((end + 15) >> 4) - c0) * D;
    for (int p0 = threadIdx.x; p0 < all; p0 += 256 * 2) {
      v4i o[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int p = min(p0 + i * 256, all - 1);
        o[i] = *(const v4i *)(src + (int64_t)(p % D) * c.page + (c0 + p / D) * 16);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int p = p0 + i * 256, d = p % D, at = (c0 + p / D) * 16;
        if (p >= all) break;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int t = at + j;
          if (t >= from0 && t < end) dst[(int64_t)(t - from0) * row + d] = T::put((float)(int8_t)((uint32_t)o[i][j >> 2] >> (8 * (j & 3))) * s);
        }
      }
    }
  }
}

// Blocks that max_new tokens behind any number of old ones can touch.
int64_t blocks_of(const CacheView &c, const BatchView &b) {
  const int64_t n = std::min(std::min<int64_t>(b.max_new, b.max_len), b.tokens);
  return std::min<int64_t>((n + c.page - 2) / c.page + 1, b.max_pages);
}

// Launches f(grid, first block) over all blocks of a batch.
template <class F>
void over_blocks(const CacheView &c, const BatchView &b, F f) {
  const int64_t blocks = blocks_of(c, b);
  for (int64_t b0 = 0; b0 < blocks; b0 += kMaxGroups)
    f(dim3((unsigned)std::min(blocks - b0, kMaxGroups), (unsigned)c.heads, (unsigned)b.requests * 2), (int)b0);
}

template <class T>
void launch_append_t(const CacheView &c, const BatchView &b, const NewKv &x, hipStream_t s) {
  const int n = append_rounds(c.page, c.dim);
  over_blocks(c, b, [&](dim3 g, int b0) {
    if (n == 1) cache_append_kernel<T, 1><<<g, kAppendThreads, 0, s>>>(c, b, x, b0);
    else if (n == 2) cache_append_kernel<T, 2><<<g, kAppendThreads, 0, s>>>(c, b, x, b0);
    else cache_append_kernel<T, 4><<<g, kAppendThreads, 0, s>>>(c, b, x, b0);
  });
}

template <class T>
void launch_read_t(const CacheView &c, const BatchView &b, const OutKv &x, hipStream_t s) {
  over_blocks(c, b, [&](dim3 g, int b0) { cache_read_kernel<T><<<g, 256, 0, s>>>(c, b, x, b0); });
}

}  // namespace

hipError_t launch_cache_append(const CacheView &c, const BatchView &b, const void *k, const void *v, int type,
                               const int64_t *stride, hipStream_t s) {
  const NewKv x{k, v, stride[0], stride[1], stride[2], stride[3]};
  if (type == PALQ_F32) launch_append_t<F32>(c, b, x, s);
  else if (type == PALQ_F16) launch_append_t<F16>(c, b, x, s);
  else launch_append_t<BF16>(c, b, x, s);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheView &c, const BatchView &b, void *k, void *v, int type, const int64_t *stride,
                             hipStream_t s) {
  const OutKv x{k, v, stride[0], stride[1], stride[2], stride[3]};
  if (type == PALQ_F32) launch_read_t<F32>(c, b, x, s);
  else if (type == PALQ_F16) launch_read_t<F16>(c, b, x, s);
  else launch_read_t<BF16>(c, b, x, s);
  return hipGetLastError();
}

}  // namespace palq
