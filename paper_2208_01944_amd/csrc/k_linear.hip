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
#include <stdlib.h>

#include "linear.h"
#include "serve_common.h"

namespace palq {

namespace {

// ------------------------------------------------------------ token quantiser
// WPR waves a row; SLABS: codes into slabs, else row by row.  A lane takes 16
// consecutive columns at a time and keeps the first kHeld such pieces in
// registers between the two looks at a row (largest magnitude, then codes): 8192
// columns of one wave, 16384 of four.  4096 rows of 8192
// bf16 (100 MB): 26 us from memory, 22 when the rows are in the caches.

template <class T, int WPR, bool SLABS>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const typename T::raw *x, int64_t rows, int cols, int64_t ld,
                                                            int kp, int8_t *codes, int64_t codes_ld, float *scales) {
  constexpr int RB = 4 / WPR, LANES = 64 * WPR, kHeld = WPR == 1 ? 8 : 4;
  __shared__ uint32_t part[4];
  const int wave = threadIdx.x >> 6, lr = threadIdx.x % LANES;
  const int64_t row = (int64_t)blockIdx.x * RB + (WPR == 1 ? wave : 0);
  const bool live = row < rows;
  const typename T::raw *xr = x + (live ? row : 0) * ld;
  float held[kHeld][16];
  uint32_t mag = 0;
  const int pieces = live ? kp / 16 : 0;
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const int p = h * LANES + lr;
    if (p < pieces) load16<T>(xr + p * 16, cols - p * 16, held[h]);
  }
#pragma unroll
  for (int h = 0; h < kHeld; ++h)
    if (h * LANES + lr < pieces)
#pragma unroll
      for (int i = 0; i < 16; ++i) mag = max(mag, mag_bits(held[h][i]));
  for (int p = kHeld * LANES + lr; p < pieces; p += LANES) {
    float v[16];
    load16<T>(xr + p * 16, cols - p * 16, v);
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
  auto put = [&](int p, const float *v) __attribute__((always_inline)) {
    const v4i o = bad ? v4i{0, 0, 0, 0} : quantize16(v, inv);
    if constexpr (SLABS) {
      const int64_t at = ((row >> 4) * (kp / 64) + (p >> 2)) * 1024 + (p & 3) * 256 + (row & 15) * 16;
      *(v4i *)(codes + at) = o;
    } else {
      int8_t *dst = codes + row * codes_ld + p * 16;
      const int n = cols - p * 16;
      if (n >= 16) {
        store_any(dst, o);
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
    load16<T>(xr + p * 16, cols - p * 16, v);
    put(p, v);
  }
}

// Codes in rows (weights, or activations given as codes) into slabs: a thread a
// piece, so a wave reads 64 bytes of 16 rows and writes a whole slab.
__global__ __launch_bounds__(256) void slab_kernel(const int8_t *x, int64_t rows, int64_t slab_rows, int cols, int64_t ld,
                                                   int kp, int8_t *out) {
  const int per = kp / 64, lane = threadIdx.x & 63;
  for (int64_t slab = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); slab < slab_rows * per; slab += (int64_t)gridDim.x * 4) {
    const int64_t rt = slab / per, row = rt * 16 + (lane & 15);
    const int k = (int)(slab - rt * per) * 64 + (lane >> 4) * 16;
    v4i o = {0, 0, 0, 0};
    if (row < rows && k < cols) {
      const int8_t *p = x + row * ld + k;
      if (k + 16 <= cols) {
        o = load_any(p);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t c = (uint8_t)p[min(i, cols - 1 - k)];
          o[i >> 2] |= k + i < cols ? (int)(c << (8 * (i & 3))) : 0;
        }
      }
    }
    *(v4i *)(out + slab * 1024 + lane * 16) = o;
  }
}

// ------------------------------------------------------------ few tokens
// A workgroup takes 16 NT channels x 16 MT tokens; its 8 waves take every eighth 64
// of k, operands straight from memory into registers, and their sums meet in LDS
// (integers: any order gives the same sum).  Bound by memory while the tokens are
// few: every wave has U blocks of both operands in flight.
constexpr int kFewWaves = 8;

// One result quad: 4 consecutive channels from n of a token.
template <class T>
__device__ __forceinline__ void put_quad(const LinearArgs &a, int64_t row, int n, v4i s, float sc) {
  if (row >= a.rows || n >= a.n_out) return;
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = min(n + i, a.n_out - 1);
    v[i] = (float)s[i] * sc * a.w_scale[c];
    if (a.bias) v[i] += a.bias[c];
  }
  typename T::raw *y = (typename T::raw *)a.y + row * a.y_ld + n;
  if (n + 4 <= a.n_out) {
    store4<T>(y, v);
  } else {
    for (int i = 0; i < 4; ++i)
      if (n + i < a.n_out) y[i] = T::put(v[i]);
  }
}
template <class T, int MT, int NT>
__global__ __launch_bounds__(64 * kFewWaves, 2) void linear_few_kernel(LinearArgs a) {
  constexpr int Q = NT * MT, U = NT + MT > 5 ? 2 : 4;
  __shared__ v4i part[kFewWaves / 2][Q][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int kb = a.kp / 64;
  const int64_t n0 = (int64_t)blockIdx.x * NT, m0 = (int64_t)blockIdx.y * MT;
  const v4i *w = (const v4i *)(a.w + n0 * kb * 1024) + lane;
  const v4i *x = (const v4i *)(a.x + m0 * kb * 1024) + lane;
  v4i acc[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[n][m] = v4i{0, 0, 0, 0};
  for (int k = wave; k < kb; k += kFewWaves * U) {
    v4i wv[U][NT], xv[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // (past the last block: the last one again, its products left out)
      const int64_t at = (int64_t)min(k + u * kFewWaves, kb - 1) * 64;
#pragma unroll
      for (int n = 0; n < NT; ++n) wv[u][n] = w[(int64_t)n * kb * 64 + at];
#pragma unroll
      for (int m = 0; m < MT; ++m) xv[u][m] = x[(int64_t)m * kb * 64 + at];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k + u * kFewWaves < kb)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[n][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][n], xv[u][m], acc[n][m], 0, 0, 0);
  }
  // the upper half of the waves through LDS into the lower, then those
  if (wave >= kFewWaves / 2)
#pragma unroll
    for (int q = 0; q < Q; ++q) part[wave - kFewWaves / 2][q][lane] = acc[q / MT][q % MT];
  __syncthreads();
  if (wave < kFewWaves / 2)
#pragma unroll
    for (int q = 0; q < Q; ++q) part[wave][q][lane] += acc[q / MT][q % MT];
  __syncthreads();
  // lane: token lane % 16, channels (lane / 16) * 4 ..
  for (int q = wave; q < Q; q += kFewWaves) {
    v4i s = part[0][q][lane];
#pragma unroll
    for (int i = 1; i < kFewWaves / 2; ++i) s += part[i][q][lane];
    const int64_t row = (m0 + q % MT) * 16 + (lane & 15);
    put_quad<T>(a, row, (int)(n0 + q / MT) * 16 + (lane >> 4) * 4, s, a.x_scale[min(row, a.rows - 1)]);
  }
}

// One token of floating values: every workgroup quantises the row by itself, into
// LDS, while its first weights are on their way; one launch instead of two.  It goes
// through its 16-channel tiles with the same row.  At most 128 registers, so that two
// workgroups on a CU keep twice the weights in flight.  A call with 4096 x 4096 weights 5.2
// us (7.5 with the quantiser in a launch of its own), 6.8 (8.8) with weights from memory;
// 8192 x 8192 12.3 (15.6), 14.8 (19.7) from memory.  (Three rows this way need 156
// registers and were slower than two launches, 17.8 us against 15.6.)
struct RawRow { const void *x; int32_t n_in; };
constexpr int kOneBytes = 16 << 10;  // at most: bytes of the row's codes

template <class T, class X>
__global__ __launch_bounds__(64 * kFewWaves, 4) void linear_one_kernel(LinearArgs a, RawRow r) {
  __shared__ __attribute__((aligned(16))) uint8_t codes[kOneBytes];
  constexpr int TH = 64 * kFewWaves, U = 8;
  __shared__ v4i part[kFewWaves][64];
  __shared__ uint32_t mags[kFewWaves];
  const typename X::raw *x = (const typename X::raw *)r.x;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, kb = a.kp / 64, tiles = (a.n_out + 15) / 16;
  v4i wv[U];
  auto fetch = [&](int tile, int k) __attribute__((always_inline)) {
    const v4i *w = (const v4i *)(a.w + (int64_t)min(tile, tiles - 1) * kb * 1024) + lane;
#pragma unroll
    for (int u = 0; u < U; ++u) wv[u] = w[(int64_t)min(k + u * kFewWaves, kb - 1) * 64];
  };
  fetch(blockIdx.x, wave);
  // largest magnitude, then codes: pieces of 16 columns, a thread every TH-th, its first
  // held between the two
  const int pieces = a.kp / 16, own = threadIdx.x;
  float held[16];
  load16<X>(x + min(own, pieces - 1) * 16, r.n_in - min(own, pieces - 1) * 16, held);
  uint32_t mag = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) mag = max(mag, mag_bits(held[j]));
  for (int p = own + TH; p < pieces; p += TH) {
    float v[16];
    load16<X>(x + p * 16, r.n_in - p * 16, v);
#pragma unroll
    for (int j = 0; j < 16; ++j) mag = max(mag, mag_bits(v[j]));
  }
  mag = wave_max(mag);
  if (lane == 0) mags[wave] = mag;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) mag = max(mag, mags[w]);
  const float s = scale_of(mag), inv = inverse_of(s);
  const v4i zero = {0, 0, 0, 0};
  if (own < pieces) *(v4i *)(codes + own * 16) = s == s ? quantize16(held, inv) : zero;
  for (int p = own + TH; p < pieces; p += TH) {
    float v[16];
    load16<X>(x + p * 16, r.n_in - p * 16, v);
    *(v4i *)(codes + p * 16) = s == s ? quantize16(v, inv) : zero;
  }
  __syncthreads();
  const uint8_t *mine = codes + (lane >> 4) * 16;  // (all 16 columns of the product are this row)
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    v4i acc = {0, 0, 0, 0};
    for (int k = wave; k < kb; k += kFewWaves * U) {
      if (k != wave) fetch(tile, k);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k + u * kFewWaves < kb)
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u], *(const v4i *)(mine + (k + u * kFewWaves) * 64), acc, 0, 0, 0);
    }
    fetch(tile + gridDim.x, wave);  // the next tile's, while the sums meet
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
      v4i sum = part[0][lane];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) sum += part[w][lane];
      put_quad<T>(a, lane & 15, tile * 16 + (lane >> 4) * 4, sum, s);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------ many tokens
// A workgroup of WC x WT waves takes 32 CT WC channels x 32 TT WT tokens, a
// wave 32 CT x 32 TT of them on v_mfma_i32_32x32x32_i8.  k goes by stages of 128:
// both operands' slabs are copied from memory straight into LDS (two stages, one
// in use, one on its way), and a wave reads the operands of the next 32 k while
// the matrix cores work on the present ones, across the stage's barrier too.  4096 rows,
// 8192 x 8192 weights: 231 us at best and 243 in the middle of 40 under the profiler, 2.38 and 2.26
// POP/s (the library's int8 product: 2.41 to 2.45; its codes come ready); the matrix cores are busy 65 % of the time at 1.7 GHz, to which
// operands of random codes bring the clock down (all-zero codes: 184 us).
// 16 bytes per lane from the buffer into LDS at `dst` (uniform) + 16 lane; in asm,
// so that the compiler does not order LDS reads after them: the stages' waits and
// barriers do.
__device__ __forceinline__ void to_lds(v4i rsrc, uint32_t dst, uint32_t voff, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(dst), "v"(voff), "s"(rsrc), "s"(soff)
               : "m0");
}
__device__ __forceinline__ v4i buffer_of(const void *base) {
  const uint64_t p = (uint64_t)base;
  return v4i{__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu)),
             -1, 0x00020000};
}
// At most N of this wave's loads in flight and its LDS reads done, then the workgroup's.
template <int N>
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

template <int WC, int WT, int CT, int TT, int S, int KB>
struct TileShape {
  static constexpr int C = 32 * CT * WC, M = 32 * TT * WT, WAVES = WC * WT;
  static constexpr int STAGE = (C + M) * 64 * KB;                   // bytes of one stage
  static constexpr int OUT = 32 * (32 * CT + 4) * 4 * WAVES;        // the epilogue's: 32 tokens of every wave
  static constexpr int LDS = S * STAGE > OUT ? S * STAGE : OUT;
  static constexpr int LOADS = (C + M) / 16 * KB / WAVES;            // 1 KB loads of a wave for a stage
  static_assert((C + M) / 16 * KB % WAVES == 0, "");
};

template <class T, int WC, int WT, int CT, int TT, int S, int KB>
__global__ __launch_bounds__(64 * WC * WT, 2) void linear_tile_kernel(LinearArgs a, int ctiles, int mtiles, int band) {
  typedef TileShape<WC, WT, CT, TT, S, KB> G;
  typedef typename T::raw R;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[G::LDS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wc = wave % WC, wt = wave / WC;

  // Workgroup i runs on XCD i % 8: each XCD takes a contiguous run of the tiles,
  // which go by bands of `band` token tiles, so that the tiles of an XCD at a
  // time share rows of both operands in its L2.
  const int tiles = ctiles * mtiles, per = (tiles + 7) / 8;
  const int t = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if (t >= tiles || (int)(blockIdx.x >> 3) >= per) return;
  const int b0 = t / (band * ctiles) * band, inb = min(band, mtiles - b0), rem = t - b0 * ctiles;
  const int ct0 = rem / inb, mt0 = b0 + rem % inb;

  const int kb = a.kp / 64, stages = kb / KB;
  const v4i rw = buffer_of(a.w + (int64_t)ct0 * (G::C / 16) * kb * 1024);
  const v4i rx = buffer_of(a.x + (int64_t)mt0 * (G::M / 16) * kb * 1024);
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
  // a stage in LDS: 16-row slabs of the channels, then of the tokens, KB slabs (64 k each) a row of them
  auto fetch = [&](int s, int slot, int i) __attribute__((always_inline)) {
    const int piece = i * G::WAVES + wave, slab = piece / KB;  // uniform
    const bool w = slab < G::C / 16;
    const uint32_t soff = (uint32_t)(((w ? slab : slab - G::C / 16) * kb + KB * s + piece % KB) * 1024);
    to_lds(w ? rw : rx, base + (uint32_t)slot * G::STAGE + piece * 1024, lane * 16, soff);
  };
  // operands of 32 k: lane l has row l % 32, 16 k from l / 32
  struct Ops { v4i w[CT], x[TT]; };
  constexpr int R32 = 2048 * KB;  // LDS bytes of 32 rows
  const int lo = (lane & 15) * 16 + (lane >> 4 & 1) * 1024 * KB + (lane >> 5) * 256;
  const int wo = lo + wc * CT * R32, xo = lo + G::C * 64 * KB + wt * TT * R32;
  auto read = [&](Ops &o, int slot, int step) __attribute__((always_inline)) {
    const uint8_t *p = lds + slot * G::STAGE + (step >> 1) * 1024 + (step & 1) * 512;
#pragma unroll
    for (int c = 0; c < CT; ++c) o.w[c] = *(const v4i *)(p + wo + c * R32);
#pragma unroll
    for (int m = 0; m < TT; ++m) o.x[m] = *(const v4i *)(p + xo + m * R32);
  };
  v16i acc[CT][TT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int m = 0; m < TT; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][m][i] = 0;
  // S stages: one in use, the next S - 1 in LDS or on their way.  A stage is asked for
  // load by load between the products of the stage S before it: asked for at once, its
  // loads keep the wave from issuing products.
  constexpr int STEPS = 2 * KB;
  Ops ops[2];
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (s < stages)
#pragma unroll
      for (int i = 0; i < G::LOADS; ++i) fetch(s, s, i);
  if (stages >= S) stage_barrier<G::LOADS * (S - 1)>();
  else stage_barrier<0>();
  read(ops[0], 0, 0);
  int slot = 0, last = S - 1;  // places of stages s and s - 1
  for (int s = 0; s < stages; ++s) {
    const int next = slot + 1 == S ? 0 : slot + 1;
    const bool more = s > 0 && s - 1 + S < stages;  // (the place of s - 1 is free since the last barrier)
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
      if (j == STEPS - 1) {
        // every read of stage s is done and stage s + 1 has landed (those after it may
        // be on their way)
        if (s + S <= stages) stage_barrier<G::LOADS * (S - 2)>();
        else stage_barrier<0>();
        if (s + 1 < stages) read(ops[0], next, 0);
      } else {
        read(ops[(j + 1) & 1], slot, j + 1);
      }
      const Ops &o = ops[j & 1];
#pragma unroll
      for (int m = 0; m < TT; ++m)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          acc[c][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.w[c], o.x[m], acc[c][m], 0, 0, 0);
          constexpr int N = CT * TT * (STEPS - 1);           // products before the last step
          const int n = (j * TT + m) * CT + c;
          if (j < STEPS - 1 && n * G::LOADS / N != (n + 1) * G::LOADS / N && more)
#pragma unroll
            for (int i = n * G::LOADS / N; i < (n + 1) * G::LOADS / N; ++i) fetch(s - 1 + S, last, i);
        }
    }
    last = slot;
    slot = next;
  }

  // 32 tokens at a time through a part of LDS that is the wave's own (the last
  // barrier came after every wave's last read), so that rows leave whole.  The
  // lane has token lane % 32 and channels 8 g + 4 (lane / 32) + i of each tile.
  constexpr int CW = 32 * CT, LD = CW + 16 / (int)sizeof(R);  // channels of the wave; a row's elements in LDS
  constexpr int E = 16 / (int)sizeof(R);                      // elements of a 16-byte store
  R *mine = (R *)(lds + wave * (G::OUT / G::WAVES));
  const int c0 = ct0 * G::C + wc * CW;
#pragma unroll
  for (int m = 0; m < TT; ++m) {
    const int64_t row0 = (int64_t)mt0 * G::M + (wt * TT + m) * 32;
    if (row0 >= a.rows) break;
    const float xs = a.x_scale[min(row0 + (lane & 31), a.rows - 1)];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int ch = c * 32 + g * 8 + (lane >> 5) * 4;
        const v4f ws = *(const v4f *)(a.w_scale + c0 + ch);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)acc[c][m][g * 4 + i] * xs * ws[i];
        if (a.bias) {
          const v4f b = *(const v4f *)(a.bias + c0 + ch);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] += b[i];
        }
        store4<T>(mine + (lane & 31) * LD + ch, v);
      }
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int PR = CW / E;  // 16-byte pieces of a row
#pragma unroll
    for (int p = 0; p < 32 * PR / 64; ++p) {
      const int piece = p * 64 + lane, r = piece / PR, e = piece % PR * E;
      const v4i o = *(const v4i *)(mine + r * LD + e);
      const int64_t row = row0 + r;
      const int n = c0 + e;
      if (row >= a.rows || n >= a.n_out) continue;
      R *y = (R *)a.y + row * a.y_ld + n;
      if (n + E <= a.n_out) {
        store_any(y, o);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (n + i < a.n_out) {
            if constexpr (sizeof(R) == 4) y[i] = __int_as_float(o[i]);
            else y[i] = (R)((uint32_t)o[i >> 1] >> (16 * (i & 1)));
          }
      }
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

template <class T, int WC, int WT, int CT, int TT, int S, int KB>
void launch_tile(const LinearArgs &a, hipStream_t s) {
  typedef TileShape<WC, WT, CT, TT, S, KB> G;
  const int ctiles = (a.n_out + G::C - 1) / G::C, mtiles = (int)((a.rows + G::M - 1) / G::M), per = (ctiles * mtiles + 7) / 8;
  linear_tile_kernel<T, WC, WT, CT, TT, S, KB><<<(unsigned)(per * 8), 64 * WC * WT, 0, s>>>(a, ctiles, mtiles, 4);
}
template <class T, int MT, int NT>
void launch_few(const LinearArgs &a, hipStream_t s) {
  linear_few_kernel<T, MT, NT><<<dim3((unsigned)((a.n_out + 16 * NT - 1) / (16 * NT)), (unsigned)((a.rows + 16 * MT - 1) / (16 * MT))),
                                 64 * kFewWaves, 0, s>>>(a);
}

// The kernel for this many rows and channels.  The largest tile that still gives
// (nearly) every CU one: operands are then read least often.  Measured with the
// quantiser, bf16, 4096 x 4096 weights: 64 rows 9.7 us on linear_few, 14.6 on 64 x 64
// tiles, 192 rows (192 tiles) 15 on either, 304 rows of 7296 to 3200 channels (250 tiles) 35
// and 25; 512 rows 22.3 on 64 x 64, 25.0 on 128 x 128; 1024 rows (a 128 x 128 tile a CU) 29.3
// with 8 waves and 4 stages of 128 k, 32.6 with 4 waves and 3 of 64, which lets three stand
// on a CU: 2048 rows 50 and 55; 4096 rows 79 on 256 x 256, 94 on 128 x 128.
enum LinearKind { kFew1, kFew2, kTile64, kTile128, kTile128Many, kTile256 };
LinearKind linear_kind(int64_t rows, int n_out) {
  auto tiles = [&](int t) { return ((n_out + t - 1) / t) * ((rows + t - 1) / t); };
  if (tiles(256) >= 192) return kTile256;
  if (tiles(128) >= 512) return kTile128Many;
  if (tiles(128) >= 256) return kTile128;
  if (rows > 32 && tiles(64) >= 160) return kTile64;
  return rows > 16 ? kFew2 : kFew1;
}

template <class T>
hipError_t launch_linear_t(const LinearArgs &a, hipStream_t s) {
  switch (linear_kind(a.rows, a.n_out)) {
    case kFew1: launch_few<T, 1, 1>(a, s); break;
    case kFew2: launch_few<T, 2, 2>(a, s); break;
    case kTile64: launch_tile<T, 2, 2, 1, 1, 4, 2>(a, s); break;
    case kTile128: launch_tile<T, 2, 4, 2, 1, 4, 2>(a, s); break;
    case kTile128Many: launch_tile<T, 2, 2, 2, 2, 3, 1>(a, s); break;
    case kTile256: launch_tile<T, 4, 2, 2, 4, 4, 1>(a, s); break;
  }
  return hipGetLastError();
}

template <class T, class X>
void launch_one_t(const LinearArgs &a, const RawRow &r, hipStream_t s) {
  const unsigned tiles = (unsigned)((a.n_out + 15) / 16);
  linear_one_kernel<T, X><<<std::min(tiles, 512u), 64 * kFewWaves, 0, s>>>(a, r);
}
template <class T>
void launch_one_x(const LinearArgs &a, const RawRow &r, int x_type, hipStream_t s) {
  if (x_type == PALQ_F32) launch_one_t<T, F32>(a, r, s);
  else if (x_type == PALQ_F16) launch_one_t<T, F16>(a, r, s);
  else launch_one_t<T, BF16>(a, r, s);
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
    for (int64_t r0 = 0; r0 < rows; r0 += 4 * kMaxGroups) {  // (slabs: fewer rows than that)
      const int64_t n = std::min(rows - r0, 4 * kMaxGroups);
      const unsigned g = (unsigned)((n + 3) / 4);
      if (slabs) quantize_rows_kernel<T, 1, true><<<g, 256, 0, s>>>((const R *)x, rows, cols, ld, kp, codes, codes_ld, scales);
      else quantize_rows_kernel<T, 1, false><<<g, 256, 0, s>>>((const R *)x + r0 * ld, n, cols, ld, kp, codes + r0 * codes_ld, codes_ld, scales + r0);
    }
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
  slab_kernel<<<(unsigned)std::min<int64_t>((slabs + 3) / 4, 1 << 16), 256, 0, s>>>(x, rows, padded_rows / 16, cols, ld, kp, out);
  return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs &a, int y_type, hipStream_t s) {
  if (y_type == PALQ_F32) return launch_linear_t<F32>(a, s);
  if (y_type == PALQ_F16) return launch_linear_t<F16>(a, s);
  return launch_linear_t<BF16>(a, s);
}

bool linear_one(int64_t rows, int32_t kp) { return rows == 1 && kp <= kOneBytes; }

hipError_t launch_linear_one(const LinearArgs &a, const void *x, int x_type, int32_t n_in, int y_type, hipStream_t s) {
  const RawRow r{x, n_in};
  if (y_type == PALQ_F32) launch_one_x<F32>(a, r, x_type, s);
  else if (y_type == PALQ_F16) launch_one_x<F16>(a, r, x_type, s);
  else launch_one_x<BF16>(a, r, x_type, s);
  return hipGetLastError();
}

const char *linear_kernel_label(int64_t rows, int n_out, int kp) {
  if (linear_one(rows, kp)) return "linear_one_kernel";
  return linear_kind(rows, n_out) <= kFew2 ? "linear_few_kernel" : "linear_tile_kernel";
}

}  // namespace palq
