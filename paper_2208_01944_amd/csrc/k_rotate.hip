// RMS norm of every head of queries and keys, and the rotation by position, in
// one pass:
//   y = x / sqrt(mean(x^2) + eps) * w,
//   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t), t = position * frequency
// for the pairs (a, b) of a head's rotating channels.
//
// Angles.  A far position times a frequency loses its fraction of a turn in fp32, so
// frequencies come as turns a position in 2^-64 of one: the product with the
// position, modulo 2^64, is the fraction, off by at most position 2^-65 turns.  Its
// upper 32 bits give the nearest quarter turn and a rest within an eighth, where
// the Taylor sums of sine (to x^9) and cosine (to x^10) end below 2^-28.
//
// Bound by memory: each element is read and written once (22.5 k tokens, 32 + 8 heads of 128
// in bf16: 91 us, 5.0 TB/s, a copy's rate; one token 3.7 us).  16 channels, 8 pairs, a
// lane, so a head is 4 to 16 lanes of one wave, pairs stay in their lane and the
// mean takes 2 to 4 steps between neighbours; a wave takes all heads of a token where
// there are tokens enough, so that angles are formed once a token.
#include <algorithm>

#include "rotate.h"

namespace palq {

namespace {

struct Turn { float c, s; };
__device__ __forceinline__ Turn turn_of(uint64_t t) {
  const int32_t v = (int32_t)(t >> 32), q = (int32_t)(((uint32_t)v + 0x20000000u) >> 30);
  const float x = (float)(int32_t)((uint32_t)v - ((uint32_t)q << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float z = x * x;
  float s = __builtin_fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  s = __builtin_fmaf(z, s, 8.33333333e-3f);
  s = __builtin_fmaf(z, s, -1.66666667e-1f);
  s = __builtin_fmaf(z * s, x, x);
  float c = __builtin_fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  c = __builtin_fmaf(z, c, -1.38888889e-3f);
  c = __builtin_fmaf(z, c, 4.16666667e-2f);
  c = __builtin_fmaf(z, c, -0.5f);
  c = __builtin_fmaf(z, c, 1.0f);
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;
  return {(q + 1) & 2 ? -a : a, q & 2 ? -b : b};
}

template <int CTRL>
__device__ __forceinline__ float other(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true));
}
// Sum over L neighbouring lanes (4, 8 or 16).
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
  x += other<0xB1>(x);
  x += other<0x4E>(x);
  if constexpr (L >= 8) x += other<0x141>(x);  // (the other four of eight, reversed)
  if constexpr (L >= 16) x += other<0x140>(x);
  return x;
}

// Channels of a lane.  HALVES: of 8 pairs, channel p with p + pairs, eight of each in a row (past the rotating
// pairs sixteen in a row).  NEIGHBOURS: 8 pairs of 2 p with 2 p + 1, sixteen in a row.  MIXED: halves that eight
// does not divide: sixteen in a row, each with its partner's value from LDS and its own angle (22.5 k tokens, 40 heads
// of 128 in bf16: 128 us for 60 pairs; 64 take 91 in HALVES, 99 in NEIGHBOURS).
enum { HALVES, NEIGHBOURS, MIXED };

template <class T>
__device__ __forceinline__ void store8(typename T::raw *p, const float *v) {
  store4<T>(p, v);
  store4<T>(p + 4, v + 4);
}
template <>
__device__ __forceinline__ void store8<F16>(uint16_t *p, const float *v) {
  v4i o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = (int)((uint32_t)F16::put(v[2 * i]) | (uint32_t)F16::put(v[2 * i + 1]) << 16);
  store_any(p, o);
}
template <>
__device__ __forceinline__ void store8<BF16>(uint16_t *p, const float *v) {
  v4i o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = (int)((uint32_t)BF16::put(v[2 * i]) | (uint32_t)BF16::put(v[2 * i + 1]) << 16);
  store_any(p, o);
}

// 16 channels of a lane in two runs of eight.
template <class T, int FORM>
struct Lane {
  float v[16];
  static __device__ __forceinline__ void runs(int lane, int pairs, int &a, int &b) {
    const bool rot = FORM == HALVES && 8 * lane < pairs;
    a = rot ? 8 * lane : 16 * lane;
    b = rot ? a + pairs : a + 8;
  }
  __device__ __forceinline__ void load(const typename T::raw *x, int lane, int pairs) {
    int a, b;
    runs(lane, pairs, a, b);
    load8<T>(x + a, v);
    load8<T>(x + b, v + 8);
  }
  __device__ __forceinline__ void store(typename T::raw *y, int lane, int pairs) const {
    int a, b;
    runs(lane, pairs, a, b);
    store8<T>(y + a, v);
    store8<T>(y + b, v + 8);
  }
};

// One wave: `each` blocks of 64 / L heads of a token, of `parts` such shares.  Queries' blocks
// come before the keys'.
template <class T, int L, int FORM>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a, int64_t first_row, int parts, int each) {
  constexpr int HEADS = 64 / L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & (L - 1), sub = (threadIdx.x & 63) / L;
  const int r = blockIdx.y;
  const bool there = 16 * lane < a.dim;
  const int mine = there ? lane : 0;
  constexpr int ANGLES = FORM == MIXED ? 16 : 8;
  __shared__ float turned[FORM == MIXED ? 4 : 1][FORM == MIXED ? 64 * 17 : 1];
  uint64_t phase[ANGLES];  // (before the request is known: one way to memory less)
#pragma unroll
  for (int i = 0; i < ANGLES; ++i) {
    const int e = ANGLES * mine + i, p = FORM == MIXED && e >= a.pairs ? e - a.pairs : e;
    phase[i] = p < a.pairs ? a.phase[p] : 0;
  }
  const Request q = request_of(a.b, r);
  const uint32_t share = blockIdx.x * 4 + wave, rank = share / (uint32_t)parts;  // (below 2^26)
  if (first_row + rank >= q.n) return;
  const int t = (int)(first_row + rank), part = (int)(share - rank * parts);
  const int64_t row = q.row0 + t;
  const int q_blocks = (a.heads[0] + HEADS - 1) / HEADS, blocks = q_blocks + (a.heads[1] + HEADS - 1) / HEADS;
  const int from = part * each, to = min(from + each, blocks);
  typedef typename T::raw Raw;
  // a block's heads, asked for before the angles, or the block before it, are ready
  Lane<T, FORM> next;
  auto load = [&](int b) __attribute__((always_inline)) {
    const int which = b >= q_blocks, h = (b - (which ? q_blocks : 0)) * HEADS + sub, hh = there && h < a.heads[which] ? h : 0;
    next.load((const Raw *)a.x[which] + row * a.x_row[which] + hh * a.x_head[which], mine, a.pairs);
  };
  if (from < to) load(from);
  int64_t pos = q.pos + (int64_t)t;
  if (a.tree.mask) {
    const Draft d = draft_of(a.b, r, a.tree.words);
    pos = (int64_t)d.old + depth_of(a.tree.mask + row * a.tree.words, a.tree.words, d.n, (int)min((int64_t)d.first + t, (int64_t)1 << 30));
  }
  float c[ANGLES], s[ANGLES];
#pragma unroll
  for (int i = 0; i < ANGLES; ++i) {
    const Turn u = turn_of((uint64_t)pos * phase[i]);
    c[i] = u.c;
    s[i] = FORM == MIXED && 16 * mine + i < a.pairs ? -u.s : u.s;
  }
  Lane<F32, FORM> w;
  int have = -1;
  const float mean = 1.0f / (float)a.dim;
  for (int b = from; b < to; ++b) {
    const int which = b >= q_blocks, h = (b - (which ? q_blocks : 0)) * HEADS + sub;
    const bool live = there && h < a.heads[which];
    Lane<T, FORM> x = next;
    if (b + 1 < to) load(b + 1);
    if (a.eps != 0.0f) {
      if (have != which && a.w[which]) w.load(a.w[which], mine, a.pairs);
      have = which;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(x.v[i], x.v[i], sum);
      sum = lanes_sum<L>(there ? sum : 0.0f);
      const float square = __builtin_fmaf(sum, mean, a.eps);
      float inv = __builtin_amdgcn_rsqf(square);
      if (__any(square == INFINITY)) {  // past fp32's range: the squares of x 2^-70, and eps 2^-140
        float less = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float z = x.v[i] * 8.470329472543003e-22f;
          less = __builtin_fmaf(z, z, less);
        }
        less = lanes_sum<L>(there ? less : 0.0f);
        const float eps = a.eps * 8.470329472543003e-22f * 8.470329472543003e-22f;
        if (square == INFINITY) inv = __builtin_amdgcn_rsqf(__builtin_fmaf(less, mean, eps)) * 8.470329472543003e-22f;
      }
      if (a.w[which]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x.v[i] = x.v[i] * inv * w.v[i];
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x.v[i] *= inv;
      }
    }
    Lane<T, FORM> y = x;
    if constexpr (FORM == MIXED) {  // (17 words for 16 channels keep banks apart)
      float *mem = turned[wave] + sub * L * 17;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 16; ++i) mem[17 * lane + i] = x.v[i];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = 16 * mine + i, o = e < a.pairs ? e + a.pairs : e - a.pairs;
        if (e < 2 * a.pairs) y.v[i] = __builtin_fmaf(x.v[i], c[i], mem[o + (o >> 4)] * s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        constexpr bool near = FORM == NEIGHBOURS;
        const int ia = near ? 2 * i : i, ib = near ? 2 * i + 1 : 8 + i;
        if (8 * mine + i < a.pairs) {
          y.v[ia] = __builtin_fmaf(x.v[ia], c[i], -(x.v[ib] * s[i]));
          y.v[ib] = __builtin_fmaf(x.v[ib], c[i], x.v[ia] * s[i]);
        }
      }
    }
    if (live) y.store((Raw *)a.y[which] + row * a.y_row[which] + h * a.y_head[which], mine, a.pairs);
  }
}

template <class T, int L>
hipError_t launch_rotate_l(const RotateArgs &a, hipStream_t s) {
  constexpr int HEADS = 64 / L;
  const int blocks = (a.heads[0] + HEADS - 1) / HEADS + (a.heads[1] + HEADS - 1) / HEADS;
  // a token's heads are shared by as many waves as it takes to have 8 on every SIMD (1024)
  const int parts = (int)std::min<int64_t>(blocks, std::max<int64_t>(1, 8192 / std::max<int64_t>(1, a.b.tokens)));
  const int each = (blocks + parts - 1) / parts, shares = (blocks + each - 1) / each;
  const int64_t most = std::max<int64_t>(1, kMaxGroups * 4 / shares - 4);  // rows of a launch
  const int64_t rows = std::min<int64_t>(a.b.max_new, a.b.tokens);
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    const int64_t n = std::min(rows - r0, most);
    const dim3 g((unsigned)((n * shares + 3) / 4), (unsigned)a.b.requests);
    if (a.interleaved || a.pairs == 0) rotate_kernel<T, L, NEIGHBOURS><<<g, 256, 0, s>>>(a, r0, shares, each);
    else if (a.pairs % 8 == 0) rotate_kernel<T, L, HALVES><<<g, 256, 0, s>>>(a, r0, shares, each);
    else rotate_kernel<T, L, MIXED><<<g, 256, 0, s>>>(a, r0, shares, each);
  }
  return hipGetLastError();
}
template <class T>
hipError_t launch_rotate_t(const RotateArgs &a, hipStream_t s) {
  return a.dim == 64 ? launch_rotate_l<T, 4>(a, s) : a.dim == 256 ? launch_rotate_l<T, 16>(a, s) : launch_rotate_l<T, 8>(a, s);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &a, int type, hipStream_t s) {
  return type == PALQ_F32 ? launch_rotate_t<F32>(a, s) : type == PALQ_F16 ? launch_rotate_t<F16>(a, s) : launch_rotate_t<BF16>(a, s);
}

}  // namespace palq
