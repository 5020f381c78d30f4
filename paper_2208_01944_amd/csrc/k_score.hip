// Log probabilities of given tokens, entropy and the k most probable tokens of a row
// of logits x, with c = scale log2(e) and M the row's largest:
//   S = sum_j 2^((x_j - M) c),  E = sum_j 2^((x_j - M) c) (x_j - M) c,
//   log p_i = (x_i - M) scale - ln S,  H = ln S - ln 2 E / S.
//
// One pass: a wave takes a row, or a part of one, 2048 logits a step.  M runs along, for
// each lane by itself, and moves only when a logit passes it by more than 2^8 (sums
// then stay far inside fp32), so most steps are an exponential and two sums an
// element; the join brings all lanes to the row's true largest, where the
// probability of a certain token loses nothing.
//
// The k largest.  A logit and its index as one 64-bit key (the value in the order of
// integers, then the index from above) have no ties, so any order of work gives the
// same list.  A bound on the keys runs along: at first the k-th of the lanes' own largest
// logits of a step, then the k-th key held.  A step's maxima are compared with it; only where
// one passes are single logits looked at, and those that pass wait in LDS until there are
// more than k by some, and are cut to the k largest.  Of n logits in random order
// k ln(n / k) pass.
//
// Large calls are bound by memory and by 11 vector instructions a logit (82 % of the time; 4096
// rows of 131071 with 20 alternatives 210 us, 5.1 TB/s, 200 without); small ones by a wave's
// chain of instructions (one such row 11.5 us in two launches, 333 rows of 1000 6.6).
#include <algorithm>
#include <float.h>

#include "score.h"

namespace palq {

namespace {

constexpr int kLongStep = 2048, kShortStep = 512;  // logits of a wave's step: 32 or 8 a lane
constexpr float kSlack = 8.0f;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ------------------------------------------------------------ keys and sorted lists
typedef uint64_t Key;  // 0: none

__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 is 0)
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t h) {
  return __uint_as_float(h & 0x80000000u ? h ^ 0x80000000u : ~h);
}
__device__ __forceinline__ Key key_of(float x, int id) { return (Key)ordered(x) << 32 | (uint32_t)~id; }
__device__ __forceinline__ int id_of(Key k) { return (int)~(uint32_t)k; }

// The value of the lane whose number differs in the bits of X.
template <int X>
__device__ __forceinline__ int across(int v) {
  if constexpr (X == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);
  else if constexpr (X == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);
  else if constexpr (X == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x1B, 0xf, 0xf, true), 0x141, 0xf, 0xf, true);  // 3, then 7
  else if constexpr (X == 8) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x140, 0xf, 0xf, true);  // 7, then 15
  else if constexpr (X == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);  // even rows of 16 everywhere, odd ones
    return threadIdx.x & 16 ? (int)r[0] : (int)r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? (int)r[0] : (int)r[1];
  }
}
template <int X>
__device__ __forceinline__ Key across(Key k) {
  return (Key)(uint32_t)across<X>((int)(k >> 32)) << 32 | (uint32_t)across<X>((int)(uint32_t)k);
}
template <int X>
__device__ __forceinline__ float across(float v) { return __int_as_float(across<X>(__float_as_int(v))); }

// One exchange: the larger stays in the lower lane where `down`.
template <int X>
__device__ __forceinline__ Key exchange(Key k, bool down) {
  const Key o = across<X>(k);
  return (k > o) == (((threadIdx.x & X) == 0) == down) ? k : o;
}
template <int X>
__device__ __forceinline__ uint32_t exchange(uint32_t k, bool down) {
  const uint32_t o = (uint32_t)across<X>((int)k), a = max(k, o), b = min(k, o);
  return ((threadIdx.x & X) == 0) == down ? a : b;
}
template <int X, class V>
__device__ __forceinline__ V merged(V k, bool down) {  // a bitonic run of 2 X lanes
  k = exchange<X>(k, down);
  if constexpr (X > 1) k = merged<X / 2>(k, down);
  return k;
}
// The wave's values, lane 0 with the largest (down) or the smallest.
template <class V>
__device__ __forceinline__ V sorted(V k, bool down) {
  const int lane = threadIdx.x & 63;
  k = merged<1>(k, ((lane & 2) == 0) == down);
  k = merged<2>(k, ((lane & 4) == 0) == down);
  k = merged<4>(k, ((lane & 8) == 0) == down);
  k = merged<8>(k, ((lane & 16) == 0) == down);
  k = merged<16>(k, ((lane & 32) == 0) == down);
  return merged<32>(k, down);
}
__device__ __forceinline__ Key lane_key(Key k, int lane) {
  return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}
__device__ __forceinline__ int rank_among(uint64_t who) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}

// The `top` largest of the keys that a wave is shown: in LDS, in no order until the end.  Alone on its
// SIMD a wave takes about eight cycles an instruction, so what counts is how few they are: keys are cut to the
// largest by sorting their 32-bit values (three instructions an exchange; a 64-bit key takes thirteen), then the
// indices of those that tie at the border; whole keys are sorted only where more than 64 wait.  Logits of -inf
// are not shown: a row with fewer others than asked for is filled up at the end.
struct TopList {
  Key bound = 0;      // keys at or below it are none of the top
  int count = 0, top;
  Key *buf;           // keys, from the first on: room for 64 and what is shown between two cuts, 128 at least

  __device__ __forceinline__ TopList(Key *b, int t) : top(t), buf(b) {}
  // The k-th largest of a value of each lane (in integers' order; 0: there is none) bounds what the first keys have to pass.
  __device__ __forceinline__ void start(uint32_t most) {
    bound = (Key)(uint32_t)__builtin_amdgcn_readlane((int)sorted(most, true), top - 1) << 32;
  }
  __device__ __forceinline__ void show(Key k) {
    const bool pass = k > bound;
    const uint64_t who = __ballot(pass);
    if (pass) buf[count + rank_among(who)] = k;
    count += __popcll(who);
  }
  // To the `top` largest.  rising: later keys of the same value are smaller (their indices are larger).
  __device__ __forceinline__ void cut(bool rising) {
    const int lane = threadIdx.x & 63;
    if (count <= top) return;
    __builtin_amdgcn_wave_barrier();
    for (int tries = 0; tries < 2 && count > 64; ++tries) {  // many: the k-th of the lanes' largest bounds them
      Key most = 0;
      for (int from = 0; from < count; from += 64) {
        const Key k = from + lane < count ? buf[from + lane] : 0;
        most = k > most ? k : most;
      }
      most = lane_key(sorted(most, true), top - 1);
      int n = 0;
      for (int from = 0; from < count; from += 64) {
        const Key k = from + lane < count ? buf[from + lane] : 0;
        const bool pass = k != 0 && k >= most;
        const uint64_t who = __ballot(pass);
        __builtin_amdgcn_wave_barrier();
        if (pass) buf[n + rank_among(who)] = k;
        n += __popcll(who);
      }
      count = n;
      __builtin_amdgcn_wave_barrier();
    }
    if (count <= 64) {
      const Key k = lane < count ? buf[lane] : 0;
      const uint32_t h = (uint32_t)(k >> 32), last = (uint32_t)__builtin_amdgcn_readlane((int)sorted(h, true), top - 1);
      uint64_t stay = __ballot(h >= last);
      if (__popcll(stay) > top) {  // of those that tie at the border, the ones with the lowest indices
        const uint64_t above = __ballot(h > last);
        const uint32_t i = h == last ? (uint32_t)k : 0;
        const uint32_t least = (uint32_t)__builtin_amdgcn_readlane((int)sorted(i, true), top - __popcll(above) - 1);
        stay = above | __ballot(i >= least);
      }
      __builtin_amdgcn_wave_barrier();
      if (stay >> lane & 1) buf[rank_among(stay)] = k;
      count = top;
      const Key b = (Key)last << 32 | (rising ? 0xffffffffu : 0u);
      bound = b > bound ? b : bound;
      return;
    }
    Key list = 0;  // sorted
    for (int from = 0; from < count; from += 64) {
      const Key k = sorted(from + lane < count ? buf[from + lane] : 0, false);
      list = merged<32>(list > k ? list : k, true);
    }
    __builtin_amdgcn_wave_barrier();
    buf[lane] = list;
    count = top;
    const Key last = lane_key(list, top - 1);
    bound = last > bound ? last : bound;
  }
  // The largest in order, one a lane (after a cut).
  __device__ __forceinline__ Key in_order() {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_wave_barrier();
    const Key k = lane < count ? buf[lane] : 0;
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < count; ++j) rank += buf[j] > k;
    if (lane < count) buf[64 + rank] = k;
    __builtin_amdgcn_wave_barrier();
    return lane < count ? buf[64 + lane] : 0;
  }
};

// ------------------------------------------------------------ sums
struct Sums {
  float m = -FLT_MAX, s = 0.0f, e = 0.0f;
  // To a maximum m2.  (Where nothing was summed the distance may be infinite; NaN stays in s.)
  __device__ __forceinline__ void move(float m2, float c) {
    const float d = fmaxf((m - m2) * c, -1e30f), w = exp2_fast(d);
    e = (e + d * s) * w;
    s *= w;
    m = m2;
  }
};

// What a row's results come from: sums under its largest, and its list of keys.
template <class T>
__device__ __forceinline__ void finish(const ScoreArgs &a, int64_t row, const Sums &z, TopList &best) {
  const int lane = threadIdx.x & 63;
  const typename T::raw *x = (const typename T::raw *)a.x + row * a.ld;
  const bool nan = z.s != z.s, none = z.s == 0.0f;
  const float shift = none ? 0.0f : logf(z.s);
  // (halves: the difference itself may be past fp32's range where its product is not)
  auto logp = [&](float x) { return nan ? __uint_as_float(0x7fc00000u) : none ? -INFINITY : (0.5f * x - 0.5f * z.m) * (2.0f * a.scale) - shift; };
  if (a.entropy && lane == 0) a.entropy[row] = nan ? __uint_as_float(0x7fc00000u) : none ? 0.0f : fmaxf(shift - kLn2 * (z.e / z.s), 0.0f);
  for (int i = lane; i < a.given; i += 64) {
    const int id = a.ids[row * a.given + i];
    a.out[row * a.given + i] = (uint32_t)id < (uint32_t)a.vocab ? logp(T::get(x[id])) : __uint_as_float(0x7fc00000u);
  }
  if (a.top == 0) return;
  int held = best.count;
  const Key list = best.in_order();
  if (lane < held) {
    a.top_ids[row * a.top + lane] = nan ? -1 : id_of(list);
    a.top_out[row * a.top + lane] = logp(value_of((uint32_t)(list >> 32)));
  }
  // the first of the tokens of -inf (in a row with NaN: any)
  for (int from = 0; held < a.top && from < a.vocab; from += 64) {
    const bool is = from + lane < a.vocab && (nan || T::get(x[from + lane]) == -INFINITY);
    const uint64_t who = __ballot(is);
    const int at = held + rank_among(who);
    if (is && at < a.top) {
      a.top_ids[row * a.top + at] = nan ? -1 : from + lane;
      a.top_out[row * a.top + at] = logp(-INFINITY);
    }
    held += __popcll(who);
  }
}

__device__ __forceinline__ Sums joined(Sums z, float most, float c) {
  z.move(most, c);
#define PALQ_STEP(X)      \
  z.s += across<X>(z.s);  \
  z.e += across<X>(z.e);
  PALQ_STEP(1) PALQ_STEP(2) PALQ_STEP(4) PALQ_STEP(8) PALQ_STEP(16) PALQ_STEP(32)
#undef PALQ_STEP
  return z;
}
__device__ __forceinline__ float wave_most(float m) {
  m = fmaxf(m, across<1>(m));
  m = fmaxf(m, across<2>(m));
  m = fmaxf(m, across<4>(m));
  m = fmaxf(m, across<8>(m));
  m = fmaxf(m, across<16>(m));
  return fmaxf(m, across<32>(m));
}

// A part's results in memory: {largest, S, E, 0}, then its keys.
__device__ __forceinline__ float *part_sums(const ScoreArgs &a, int64_t unit) { return a.part + unit * 4; }
__device__ __forceinline__ Key *part_keys(const ScoreArgs &a, int64_t units, int64_t unit) { return (Key *)(a.part + units * 4) + unit * a.top; }

// A wave takes a row, or, of rows that are split, four waves one of the row's `splits` parts.
template <class T, bool TOP, int STEP>
__global__ __launch_bounds__(256) void score_kernel(ScoreArgs a, int64_t first_row, int64_t rows) {
  typedef typename T::raw Raw;
  constexpr int VEC = 16 / sizeof(Raw), U = STEP / (64 * VEC), kStep = STEP;
  // A long step's runs of 16 bytes whose largest passes the bound wait in a queue, with their first indices, so that
  // the few logits that pass are looked at 64 at a time; a short step looks at each of a lane's 8 (1500 rows of 50000: 49 us,
  // 79 so in long steps; one row: 12.0 us with the queue, 11.9).
  constexpr bool QUEUED = TOP && STEP == kLongStep;
  __shared__ v4i queue[4][QUEUED ? 64 * U : 1];
  __shared__ int ids[4][QUEUED ? 64 * U : 1];
  __shared__ Key bufs[TOP ? 4 : 1][QUEUED ? 256 : TOP ? 64 + STEP : 1];
  __shared__ int counts[4];
  __shared__ v4f sums[4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const bool team = a.splits > 0;
  const int64_t unit = team ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  if (unit >= (team ? rows * a.splits : rows)) return;
  const int64_t row = first_row + (team ? unit / a.splits : unit);
  const int split = team ? (int)(unit % a.splits) * 4 + wave : 0;
  // places count from the last multiple of 16 bytes at or before the row: logit i at place from + i
  const Raw *x = (const Raw *)a.x + row * a.ld;
  const int from = (int)((uintptr_t)x & 15) / (int)sizeof(Raw), to = from + a.vocab;
  x -= from;
  const float c = a.scale * kLog2e;
  const int last = min((to + kStep - 1) / kStep, (split + 1) * a.each);

  v4i now[U], next[U];
  auto load = [&](int step, v4i *d) __attribute__((always_inline)) {
    const int p0 = step * kStep;
    if (p0 >= from && p0 + kStep <= to) {
#pragma unroll
      for (int u = 0; u < U; ++u) d[u] = *(const v4i *)(x + p0 + (u * 64 + lane) * VEC);
    } else {  // the row's ends: single logits, and -inf outside
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = p0 + (u * 64 + lane) * VEC;
        if (p >= from && p + VEC <= to) {
          d[u] = *(const v4i *)(x + p);
        } else {
          Raw r[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) r[i] = p + i >= from && p + i < to ? x[p + i] : T::put(-INFINITY);
          __builtin_memcpy(&d[u], r, 16);
        }
      }
    }
  };
  auto get = [&](const v4i &d, int i) __attribute__((always_inline)) {
    if constexpr (VEC == 4) return __int_as_float(d[i]);
    else return T::get((uint16_t)((uint32_t)d[i >> 1] >> (i & 1) * 16));
  };
  Sums z;
  float most = -INFINITY;
  TopList best(bufs[TOP ? wave : 0], a.top);
  int step = split * a.each;
  if (step < last) load(step, now);
  for (bool begun = false; step < last; ++step, begun = true) {
    if (step + 1 < last) load(step + 1, next);
    float mx[U], m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      mx[u] = get(now[u], 0);
#pragma unroll
      for (int i = 1; i < VEC; ++i) mx[u] = fmaxf(mx[u], get(now[u], i));
      m = fmaxf(m, mx[u]);
    }
    most = fmaxf(most, m);
    if (__any((m - z.m) * c > kSlack)) z.move(fmaxf(z.m, m), c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float s = 0.0f, e = 0.0f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float t = (get(now[u], i) - z.m) * c, w = exp2_fast(t);
        s += w;
        e = __builtin_fmaf(w, fmaxf(t, -200.0f), e);  // (w = 0 from 2^-150 on: -inf must not meet it)
      }
      z.s += s;
      z.e += e;
    }
    if constexpr (TOP) {
      const int id0 = step * kStep - from;
      if (!begun) best.start(m == -INFINITY ? 0 : ordered(m));
      // A logit of the bound's value is below it if its index is larger, as all of this step's are if the first is
      // (the first bound has no index: it counts as the largest).
      uint32_t h = (uint32_t)(best.bound >> 32);
      if ((uint32_t)id_of(best.bound) >= (uint32_t)id0) h -= h == 0x80000000u ? 2 : 1;
      const float pass = best.bound ? value_of(h) : -INFINITY;
      const int id1 = id0 + lane * VEC;
      if (!QUEUED && __any(m > pass)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float v = get(now[u], i);
            if (__any(v > pass)) best.show(v > pass ? key_of(v, id1 + u * 64 * VEC + i) : 0);  // (outside the row there is only -inf)
          }
        if (best.count > min(64, best.top + 24)) best.cut(true);
      }
      if (QUEUED && __any(m > pass)) {
        int n = 0;  // runs in the queue
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const bool hit = mx[u] > pass;
          const uint64_t who = __ballot(hit);
          if (who == 0) continue;
          if (hit) {
            const int at = n + rank_among(who);
            queue[wave][at] = now[u];
            ids[wave][at] = id1 + u * 64 * VEC;
          }
          n += __popcll(who);
        }
        __builtin_amdgcn_wave_barrier();
        for (int e = lane; e - lane < n * VEC; e += 64) {  // (in the order of their indices)
          const int at = min(e, n * VEC - 1);
          const float v = T::get(((const Raw *)queue[wave])[at]);
          best.show(e == at && v > pass ? key_of(v, ids[wave][at / VEC] + at % VEC) : 0);
          if (best.count > 64) best.cut(true);
        }
        __builtin_amdgcn_wave_barrier();
        if (best.count > min(64, best.top + 24)) best.cut(true);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = next[u];
  }
  if constexpr (TOP) best.cut(true);
  most = fmaxf(wave_most(most), -FLT_MAX);
  z = joined(z, most, c);
  if (team) {  // the four waves' results to the first
    if (lane == 0) sums[wave] = v4f{z.m, z.s, z.e, 0.0f};
    if (TOP && lane == 0) counts[wave] = best.count;
    __syncthreads();
    if (wave > 0) return;
    float m = z.m;
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, sums[w][0]);
    z.move(m, c);
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      Sums o;
      o.m = sums[w][0];
      o.s = sums[w][1];
      o.e = sums[w][2];
      o.move(m, c);
      z.s += o.s;
      z.e += o.e;
    }
    if constexpr (TOP) {
      Key k[4];
      uint32_t h = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int from = (lane + 16 * w) & 63;  // (over all lanes, so that their largest bound the rest)
        k[w] = from < counts[w] ? bufs[w][from] : 0;
        h = max(h, (uint32_t)(k[w] >> 32));
      }
      best.start(h);
      best.count = 0;
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int w = 0; w < 4; ++w) best.show(k[w]);
      best.cut(false);
    }
  }
  if (a.splits <= 1) {
    finish<T>(a, row, z, best);
    return;
  }
  if (lane == 0) *(v4f *)part_sums(a, unit) = v4f{z.m, z.s, z.e, 0.0f};
  if (lane < a.top) part_keys(a, rows * a.splits, unit)[lane] = lane < best.count ? best.buf[lane] : 0;
}

// A wave a row: the parts under one maximum, the largest of their keys.
template <class T, bool TOP>
__global__ __launch_bounds__(256) void score_join_kernel(ScoreArgs a, int64_t first_row, int64_t rows) {
  constexpr int N = 24;  // keys of a lane at a time: 76 parts of 20
  __shared__ Key bufs[TOP ? 4 : 1][TOP ? 64 + 64 * N : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + wave;
  if (r >= rows) return;
  const float c = a.scale * kLog2e;
  TopList best(bufs[TOP ? wave : 0], a.top);
  if constexpr (TOP) {
    const Key *keys = part_keys(a, rows * a.splits, r * a.splits);
    const int n = a.splits * a.top;
    for (int k0 = 0; k0 < n; k0 += 64 * N) {
      Key k[N];
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = k0 + i * 64 + lane;
        k[i] = at < n ? keys[at] : 0;
      }
      if (k0 == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) most = max(most, (uint32_t)(k[i] >> 32));
        best.start(most);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) best.show(k[i]);
      best.cut(false);
    }
  }
  Sums z;
  float most = -FLT_MAX;
  for (int s = lane; s < a.splits; s += 64) most = fmaxf(most, part_sums(a, r * a.splits + s)[0]);
  most = wave_most(most);
  for (int s = lane; s < a.splits; s += 64) {
    const v4f p = *(const v4f *)part_sums(a, r * a.splits + s);
    Sums o;
    o.m = p[0];
    o.s = p[1];
    o.e = p[2];
    o.move(most, c);
    z.s += o.s;
    z.e += o.e;
  }
  z.m = most;
  z = joined(z, most, c);
  finish<T>(a, first_row + r, z, best);
}

template <class T, bool TOP>
hipError_t launch_score_t(const ScoreArgs &a, hipStream_t s) {
  const int64_t most = a.splits ? kMaxGroups / a.splits : kMaxGroups * 4;  // rows of a launch
  for (int64_t r0 = 0; r0 < a.rows; r0 += most) {
    const int64_t n = std::min(a.rows - r0, most);
    const unsigned g = (unsigned)(a.splits ? n * a.splits : (n + 3) / 4);
    if (a.step == kShortStep) score_kernel<T, TOP, kShortStep><<<g, 256, 0, s>>>(a, r0, n);
    else score_kernel<T, TOP, kLongStep><<<g, 256, 0, s>>>(a, r0, n);
    if (a.splits > 1) score_join_kernel<T, TOP><<<(unsigned)((n + 3) / 4), 256, 0, s>>>(a, r0, n);
  }
  return hipGetLastError();
}

}  // namespace

void score_plan(ScoreArgs &a, int cus) {
  auto steps = [&](int step) { return (int32_t)(((int64_t)a.vocab + 15 + step - 1) / step); };
  // A wave for each row where those fill every SIMD four times, or rows are a step.  (4096 rows of 32000: 70 us; four waves
  // for each row, and a list for each wave, would be 88.)
  if (steps(kShortStep) < 2 || a.rows >= (int64_t)16 * cus || (a.rows >= (int64_t)4 * cus && steps(kLongStep) < 2)) {
    a.step = steps(kShortStep) < 2 ? kShortStep : kLongStep;
    a.splits = 0;
    a.each = steps(a.step);
    return;
  }
  // Else workgroups of four waves, in long steps where one for each wave still puts a wave on every SIMD, or two for each
  // make one workgroup; one workgroup a row, without a join, from two rows a CU on and up to 16 steps (one row of 4000,
  // 8000 and 16000: 7.6, 7.6 and 9.6 us, in parts 10.4, 11.3 and 11.2), else up to four waves a SIMD.
  const int64_t total = a.rows * steps(kLongStep);
  a.step = total >= (int64_t)4 * cus || (steps(kLongStep) >= 3 && steps(kLongStep) <= 8) ? kLongStep : kShortStep;
  const int32_t n = steps(a.step);
  const int64_t waves = a.rows >= (int64_t)2 * cus || n <= 16 ? 4 : std::max<int64_t>(4, std::min<int64_t>(n, (int64_t)16 * cus / a.rows));
  a.each = (int32_t)std::max<int64_t>((n + (waves == 4 ? 3 : waves / 2)) / waves, (n + 511) / 512);
  a.splits = (n + 4 * a.each - 1) / (4 * a.each);
}

size_t score_work_bytes(const ScoreArgs &a) {
  return a.splits <= 1 ? 0 : (size_t)a.rows * a.splits * (16 + 8 * (size_t)a.top);
}

hipError_t launch_score(const ScoreArgs &a, int type, hipStream_t s) {
  switch (type) {
    case PALQ_F32: return a.top ? launch_score_t<F32, true>(a, s) : launch_score_t<F32, false>(a, s);
    case PALQ_F16: return a.top ? launch_score_t<F16, true>(a, s) : launch_score_t<F16, false>(a, s);
    default: return a.top ? launch_score_t<BF16, true>(a, s) : launch_score_t<BF16, false>(a, s);
  }
}

}  // namespace palq
