// Types and helpers shared by the 8-bit transformer operators (k_linear.hip,
// k_cache.hip, k_attend.hip).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "conv_common.h"
#include "palq.h"

namespace palq {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// The quantiser of the 8-bit operators, in fp32: s = max(a fl(1/127), 2^-100),
// a the largest magnitude, code = clamp(rint(x fl(1/s)), -127, 127).  The floor
// keeps 1/s, and the products of a scale's reciprocal with sums of
// probabilities, finite.  A block with an element that is not finite has scale
// NaN and codes 0.
constexpr float kInv127 = 1.0f / 127.0f;
constexpr float kScaleFloor = 7.88860905e-31f;  // 2^-100

// a as the bits of |x|: their order as integers is the order of the values,
// with inf and then NaN above every number, so a maximum of integers cannot
// lose a NaN.
__device__ __forceinline__ uint32_t mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(uint32_t mag) {
  return mag >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__uint_as_float(mag) * kInv127, kScaleFloor);
}
// inv = 1 / s, or 0 where s is NaN
__device__ __forceinline__ float inverse_of(float s) { return s == s ? 1.0f / s : 0.0f; }
__device__ __forceinline__ int code_of(float x, float inv) {
  const float t = x * inv;
  return (int)fminf(fmaxf(__builtin_rintf(t), -127.0f), 127.0f);  // NaN (x not finite, inv 0): fmaxf gives -127
}

// Element types of tensors in memory.
struct F32 { typedef float raw; static __device__ __forceinline__ float get(raw v) { return v; }
             static __device__ __forceinline__ raw put(float v) { return v; } };
struct F16 { typedef uint16_t raw;
             static __device__ __forceinline__ float get(raw v) { return (float)__builtin_bit_cast(_Float16, v); }
             static __device__ __forceinline__ raw put(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); } };
struct BF16 { typedef uint16_t raw;
              static __device__ __forceinline__ float get(raw v) { return __uint_as_float((uint32_t)v << 16); }
              static __device__ __forceinline__ raw put(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); } };

// 16 and 8 bytes at any address: the hardware's vector loads and stores need no
// alignment, and odd row lengths must not cost a load for every element.
__device__ __forceinline__ v4i load_any(const void *p) {
  v4i v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
template <class V>
__device__ __forceinline__ void store_any(void *p, V v) { __builtin_memcpy(p, &v, sizeof(V)); }

// Four consecutive values to p.
template <class T>
__device__ __forceinline__ void store4(typename T::raw *p, const float *v) {
  if constexpr (sizeof(typename T::raw) == 4) {
    store_any(p, v4f{v[0], v[1], v[2], v[3]});
  } else {
    const uint32_t a = (uint32_t)T::put(v[0]) | (uint32_t)T::put(v[1]) << 16;
    const uint32_t b = (uint32_t)T::put(v[2]) | (uint32_t)T::put(v[3]) << 16;
    store_any(p, v2i{(int)a, (int)b});
  }
}

// Eight consecutive values from p.
template <class T>
__device__ __forceinline__ void load8(const typename T::raw *p, float *v) {
  const v4i a = load_any(p);
  if constexpr (sizeof(typename T::raw) == 4) {
    const v4i b = load_any(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __int_as_float(a[i]);
      v[4 + i] = __int_as_float(b[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = T::get((uint16_t)((uint32_t)a[i] & 0xffffu));
      v[2 * i + 1] = T::get((uint16_t)((uint32_t)a[i] >> 16));
    }
  }
}

// Sixteen consecutive values from p, of which the first n exist (the others are
// 0; n may be 0 or less, and p[n - 1] is there in any case).
template <class T>
__device__ __forceinline__ void load16(const typename T::raw *p, int n, float *v) {
  if (n >= 16) {
    load8<T>(p, v);
    load8<T>(p + 8, v + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {  // (every load in flight: none waits for a condition)
      const float x = T::get(p[min(i, n - 1)]);
      v[i] = i < n ? x : 0.0f;
    }
  }
}

// Sixteen codes as one 16-byte piece.
__device__ __forceinline__ v4i quantize16(const float *v, float inv) {
  v4i o;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)code_of(v[4 * q + i], inv) & 0xffu) << (8 * i);
    o[q] = (int)w;
  }
  return o;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t a) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, off));
  return a;
}

// A launch has fewer than 2^32 threads along x: of 256 threads, this many workgroups at most.
constexpr int64_t kMaxGroups = ((int64_t)1 << 24) - 1;

// A paged cache and a batch of requests as the kernels take them
// (include/palq.h has their meaning).
struct CacheView {
  int8_t *k, *v;
  float *ks, *vs;
  int32_t pages, heads, dim, page, shift;  // page = 1 << shift tokens
};
struct BatchView {
  const int32_t *table, *lens, *starts;
  int32_t requests, max_pages, max_new;
  int64_t tokens, max_len;
  int32_t rows, limit;  // tokens, and the most that a request holds, in 32 bits
};

// One request: `n` ragged rows from row0 on, at positions pos, pos + 1, .., and `len`
// tokens.  Whatever the arrays hold, len stays inside the table and the rows
// inside the tensors; what is left out (rows or tokens past the bounds) does not
// move the others: row i of the tensors is at lens[r] - starts[r + 1] + i.  In 32 bits,
// so that it stays in scalar registers; pos wraps round only where n or len is 0.
struct Request { int64_t row0; int32_t n, len, pos; };
constexpr int64_t kMaxTokens = ((int64_t)1 << 31) - 1024;  // so that the tiles that are asked for past a request's end have 32-bit places
__device__ __forceinline__ Request request_of(const BatchView &b, int r) {
  const int32_t s0 = b.starts[r], s1 = b.starts[r + 1], all = b.lens[r];
  const int32_t row0 = max(s0, 0), end = min(s1, b.rows);
  Request q;
  q.row0 = row0;
  q.n = end > row0 ? max(0, min(end - row0, b.max_new + min(s0, 0))) : 0;  // (max_new counts from starts[r])
  q.len = max(0, min(all, b.limit));
  q.pos = (int32_t)((uint32_t)all - (uint32_t)s1 + (uint32_t)row0);
  return q;
}

// The drafted tokens of a request (its new rows) as a tree: row i's bit b stands for new
// token b, counted from starts[r].
struct TreeView { const uint64_t *mask; int32_t words; };  // [tokens][words]; null: no tree
struct Draft {
  int32_t old;    // tokens before the first new one (below 0: as many new ones lie before the request)
  int32_t n;      // new tokens that have a bit
  int32_t first;  // index of the first row that is inside the tensors
};
__device__ __forceinline__ Draft draft_of(const BatchView &b, int r, int words) {
  const int64_t s0 = b.starts[r], s1 = b.starts[r + 1], all = b.lens[r], n = s1 - s0, bits = 64 * words;
  const int64_t old = all - n;
  return {(int32_t)(old < -(1 << 30) ? -(1 << 30) : old > 0x7fffffff ? 0x7fffffff : old), (int32_t)(n < 0 ? 0 : n > bits ? bits : n),
          (int32_t)(s0 < 0 ? -s0 > (1 << 30) ? 1 << 30 : -s0 : 0)};
}
// How many of the n new tokens a row sees besides itself (new token `self`).
__device__ __forceinline__ int depth_of(const uint64_t *mask, int words, int n, int self) {
  int depth = 0;
  for (int w = 0; w < words; ++w) {
    const int left = n - 64 * w, me = self - 64 * w;
    uint64_t x = left >= 64 ? mask[w] : left <= 0 ? 0 : mask[w] & (((uint64_t)1 << left) - 1);
    if (me >= 0 && me < 64) x &= ~((uint64_t)1 << me);
    depth += __popcll(x);
  }
  return depth;
}

}  // namespace palq
