// Attention over the paged 8-bit cache:
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j,  k_j = code ks[block], v_j = code vs[block]
// over the tokens j that query i sees (its own position and earlier ones, or a
// window of them, or all; with a window, the request's first tokens too; of a tree of
// drafted tokens, those whose bit its mask has).
//
// Scores and sums are fp32.  The codes are exact in fp16, so q is the only
// operand that is rounded: each row is scaled by a power of two that brings its
// largest element to [2^14, 2^15), the top of fp16's range, so that bf16 values (8 bits)
// stay exact down to 2^-31 of the row's largest and fp16 values (11 bits) down to 2^-28;
// the scale of a block multiplies the finished dot product.  Probabilities are rounded to
// fp16 (11 bits) as the second product's operand.
//
// Value scales.  Blocks of any scale meet in one row, and a block whose scale one large
// element sets may hold zeros in every other channel, so weights must keep their bits
// beside a block of far larger scale.  vs = 2^(U + a) r: U, the unit that the
// accumulators are in, follows the tiles' largest scales (within 4 powers of two of each
// tile's, but at least 2^-72 of the largest so far: fp32 holds that); 2^a, -24 <= a <= 4,
// goes into the fp16 codes, exactly, in the operation that converts them; what is left, r
// in [1, 2), rides in the softmax's exponent: with u_j = log2 r, w_j = exp2(s_j + u_j - M),
// M a running maximum, out = 2^U sum w_j (code_j 2^a) / L, L = sum w_j / r, and w stays
// in fp16's range (at most 2^8 above the largest: kSlack).  Where a tile of 64 tokens has
// one scale (prompts, pages of a tile or more), U lies 0 to 4 below it and r in [1, 32).
// Blocks within 2^20 of their tile's largest scale, and tiles within 2^72 of all others,
// lose nothing; below, r falls under 1, and fp16 has 11 bits of the weight for 14 powers
// of two more.  A scale of 0 counts in L (r is held at 2^-64) and adds nothing else.
//
// Matrix layout.  S^T = K Q^T with v_mfma_f32_16x16x32_f16: a lane ends up with
// scores of one query (lane % 16) and, row 4 c + i of subtile j standing for
// token 16 c + 4 j + i (c = lane / 16), with 16 consecutive tokens: all of one
// page, with one pair of scales, and in the order in which O^T = V^T P^T takes
// them as its second operand.  So probabilities never leave their lane, and V,
// stored channel by channel, is read 16 tokens at a time.
//
// Two kernels.  attend_rows_kernel: few rows, everything in registers, tokens cut
// over waves and workgroups; bound by the cache's bytes.  attend_tile_kernel:
// prompts, 128 rows a workgroup over tiles in LDS; bound by the softmax's vector
// instructions and the products in turn.
#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "cache_index.h"

namespace palq {

namespace {

// 4 codes of a word as fp16: bytes of x + 128 under the exponent of 1024 are
// 1024 + 128 + x, exactly.
__device__ __forceinline__ void codes_h4(uint32_t x, h2 &a, h2 &b) {
  const uint32_t u = x ^ 0x80808080u;
  const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
  a = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
  b = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
}
// The same times a power of two m (2^-24 to 2^4, or 0; n = -1152 m): as many operations.
__device__ __forceinline__ void codes_h4(uint32_t x, h2 m, h2 n, h2 &a, h2 &b) {
  const uint32_t u = x ^ 0x80808080u;
  a = __builtin_elementwise_fma(__builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)), m, n);
  b = __builtin_elementwise_fma(__builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)), m, n);
}
__device__ __forceinline__ h8 codes_h8(uint32_t x, uint32_t y, uint32_t mm, uint32_t nn) {
  const h2 m = __builtin_bit_cast(h2, mm), n = __builtin_bit_cast(h2, nn);
  h2 a, b, c, d;
  codes_h4(x, m, n, a, b);
  codes_h4(y, m, n, c, d);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ h8 codes_h8(uint32_t x, uint32_t y) {
  h2 a, b, c, d;
  codes_h4(x, a, b);
  codes_h4(y, c, d);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kLog2e = 1.44269504088896340736f;  // (times the row's factor first: scales near 2^128 are numbers too)

// The running maximum moves only when a score passes it by more than 2^8: weights
// up to 2^8 lose nothing in fp16 or fp32, and most tiles then leave the outputs'
// accumulators alone.
constexpr float kSlack = 8.0f;

// The unit 2^u of the output accumulators (kNoUnit before the first scale).
constexpr int kNoUnit = -512;
__device__ __forceinline__ int exponent_of(float s) {  // of a normal number; kNoUnit of 0, inf and NaN
  const int e = (int)(__float_as_uint(s) >> 23) & 255;
  return e == 0 || e == 255 ? kNoUnit : e - 127;
}
struct Unit {
  int u = kNoUnit, top = kNoUnit;
  // To n, or to 2^-72 of the largest scale so far where that is more (2^72, weights of 2^13, codes of 2^7 and
  // 2^31 tokens: sums stay in fp32); e: the tile's largest exponent.
  __device__ __forceinline__ void move(int n, int e) {
    top = max(top, e);
    u = max(n, top - 72);
  }
  // Keeps e within [u - 4, u + 4].
  __device__ __forceinline__ bool leaves(int e) const { return e != kNoUnit && (e > u + 4 || e < u - 4); }
};
// Scale over unit, q = vs / 2^U: its power of two 2^a goes into the codes (two halves of m, and of n = -1152 m), the
// rest into the exponent (u, and 1 / r).  whole: all of it goes into the exponent.
struct ValueScale { float u, rv; uint32_t m, n; };
__device__ __forceinline__ ValueScale value_scale(float q, bool whole = false) {
  const float pow2 = fminf(fmaxf(__uint_as_float(__float_as_uint(q) & 0x7f800000u), 5.9604645e-8f), 16.0f);  // 2^-24 .. 2^4
  const float p = whole ? 1.0f : pow2;
  const float r = q * __builtin_amdgcn_rcpf(p), l = __builtin_amdgcn_logf(r), u = l < -64.0f ? -64.0f : l;  // (NaN stays)
  const float f = q == 0.0f ? 0.0f : p;
  const h2 m = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(f, f)), n = m * h2{(_Float16)-1152.0f, (_Float16)-1152.0f};
  return {u, exp2_fast(-u), __builtin_bit_cast(uint32_t, m), __builtin_bit_cast(uint32_t, n)};
}

// One row's reach: tokens [lo, hi).
struct Reach { int lo, hi; };
__device__ __forceinline__ Reach reach_of(const AttendArgs &a, const Request &q, int t) {
  const int pos = q.pos + t;
  Reach s{0, q.len};
  if (a.causal) {
    s.hi = max(0, min(q.len, pos + 1));
    if (a.window > 0 && pos >= a.window) s.lo = pos - a.window + 1;  // (pos may be negative, the window near 2^31)
  }
  return s;
}

// What a row sees.  RANGE: a range.  SINKS: with the first tokens before it, of which
// tiles come first, so that what lies between is never read.  TREE: a range (and first
// tokens) of the tokens before the new ones, and the new ones by bits.
enum { RANGE, SINKS, TREE };

// A tree's rows go neither forward nor back, so their common bounds come from the
// least and the largest position that a row can have.
struct Canopy {
  int old;            // first new token (below 0: the new ones up to there lie before the request)
  int context, end;   // tokens before the new ones, and before the first that no bit stands for
  int low, high;      // least and largest first token of a row's range
};
__device__ __forceinline__ Canopy canopy_of(const AttendArgs &a, const Request &q, int r) {
  const Draft d = draft_of(a.b, r, a.tree.words);
  Canopy c{max(d.old, -64 * PALQ_TREE_WORDS), max(0, min(d.old, q.len)), (int)max((int64_t)0, min((int64_t)d.old + d.n, (int64_t)q.len)), 0, 0};
  if (a.window > 0) {
    c.low = (int)max((int64_t)0, (int64_t)d.old - a.window + 1);
    c.high = (int)min(max((int64_t)0, (int64_t)d.old + d.n - a.window + 1), (int64_t)0x7fffffff);  // (a row without a bit may see all n)
  }
  return c;
}
// Row t's range.
__device__ __forceinline__ Reach branch_of(const AttendArgs &a, const Request &q, const Canopy &cp, int r, int t) {
  Reach s{0, cp.context};
  if (a.window > 0) {
    const Draft d = draft_of(a.b, r, a.tree.words);
    const int depth = depth_of(a.tree.mask + (q.row0 + t) * a.tree.words, a.tree.words, d.n, (int)min((int64_t)d.first + t, (int64_t)1 << 30));
    s.lo = (int)min(max((int64_t)0, (int64_t)d.old + depth - a.window + 1), (int64_t)0x7fffffff);
  }
  return s;
}
// Bits b .. b + 15 of a row of masks; 0 outside its words.
__device__ __forceinline__ uint32_t bits16(const uint64_t *mask, int words, int b) {
  if (b <= -16 || b >= 64 * words) return 0;
  const uint32_t *w = (const uint32_t *)mask;
  const int i = b >> 5;
  const uint32_t lo = i >= 0 ? w[i] : 0, hi = i + 1 < 2 * words ? w[i + 1] : 0;
  return __builtin_amdgcn_alignbit(hi, lo, b & 31) & 0xffffu;
}
// The lowest n bits of 16.
__device__ __forceinline__ uint32_t first16(int n) { return n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1; }
// Which of the 16 tokens from tok on a row sees that has the range [lo, hi); of sinks, and of a tree's new tokens.
__device__ __forceinline__ uint32_t seen16(const AttendArgs &a, const Request &q, int tok, int lo, int hi, const Canopy &cp, const uint64_t *mask) {
  uint32_t m = (first16(hi - tok) & ~first16(lo - tok)) | first16(min(a.sinks, hi) - tok);
  if (mask && tok + 16 > cp.old) m |= bits16(mask, a.tree.words, tok - cp.old) & first16(cp.end - tok);
  return m;
}

// The tiles of 64 tokens that a block of rows takes, by number: RANGE: their places; else tiles_seen's.
template <int SEES>
struct Tiles {
  int first, count;
  TileOrder order{0, 0, 0};
  __device__ __forceinline__ Tiles(const AttendArgs &a, int lo, int hi) {
    if constexpr (SEES == RANGE) {
      first = lo >> 6;
      count = hi > lo ? ((hi + 63) >> 6) - first : 0;
    } else {
      order = tiles_seen(lo, hi, a.sinks);
      first = 0;
      count = order.count;
    }
  }
  __device__ __forceinline__ int at(int i) const { return SEES == RANGE ? i : order.at(i); }
};

// The power of two that brings a row's largest magnitude (its bits) to [2^14, 2^15),
// and its inverse.  A row with inf or NaN: 0, so that inf 0 = NaN reaches all of
// its scores.
struct RowScale { float in, out; };
__device__ __forceinline__ RowScale row_scale(uint32_t mag) {
  const int e = (int)(mag >> 23), b = min(max(e, 15), 254);
  return {e == 255 ? 0.0f : __uint_as_float((uint32_t)(268 - b) << 23), __uint_as_float((uint32_t)(b - 14) << 23)};
}

template <class T>
__device__ __forceinline__ float low(int w) { return T::get((uint16_t)((uint32_t)w & 0xffffu)); }
template <class T>
__device__ __forceinline__ float high(int w) { return T::get((uint16_t)((uint32_t)w >> 16)); }
template <class T, int N>
__device__ __forceinline__ uint32_t largest(const v4i *raw) {
  uint32_t mag = 0;
#pragma unroll
  for (int s = 0; s < N; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) mag = max(mag, max(mag_bits(low<T>(raw[s][i])), mag_bits(high<T>(raw[s][i]))));
  return mag;
}
template <class T>
__device__ __forceinline__ h8 scaled(v4i raw, float f) {
  h8 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = (_Float16)(low<T>(raw[i]) * f);
    o[2 * i + 1] = (_Float16)(high<T>(raw[i]) * f);
  }
  return o;
}

__device__ __forceinline__ float other_half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// (of the lane 16 on, or before, in the same half)
__device__ __forceinline__ float other_row_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// ------------------------------------------------------------ few rows
// NQ tiles of 16 (query, head) rows a wave, W waves a workgroup (rows_waves), each wave every
// W-th tile of 64 tokens; the waves join in LDS, splits in attend_join_kernel.
// Operands go from memory straight into registers, one tile ahead.  32 requests of 2047
// to 16384 tokens, 8 heads of 128, group 4 (605 MB of codes): 117 us, 5.2 TB/s (a
// plain read of memory reaches 6.1); 4 requests, 5 tokens, window 8191: 21 us.  With sinks, 32
// single tokens of a window of 4096: 50 us, 5.2 TB/s; 8 drafts of 11 to 25 tokens, heads of 96 in groups of
// 7, behind 4095: 31 us, where 144 of 256 CUs have rows and their SIMDs are 70 % in vector instructions,
// 17 % in products.
template <class T, int D, int NQ, int SEES, int W>
__global__ __launch_bounds__(64 * W, D < 256 ? 2 : 1) void attend_rows_kernel(AttendArgs a) {
  constexpr int KS = D / 32, DT = D / 16, OLD = D + 4;
  constexpr int CH = D % 64 == 0 ? 16 : 8;  // consecutive channels of a key that a lane loads at once
  __shared__ float sm[W][NQ * 16], sl[W][NQ * 16];
  __shared__ int su[W];
  __shared__ __attribute__((aligned(16))) float so[W][16 * OLD];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, c = lane >> 4;
  const CacheView &cv = a.c;
  const int heads = cv.heads;
  int h = blockIdx.y, r = blockIdx.z, split = blockIdx.x % a.splits, rt = blockIdx.x / a.splits;
  if constexpr (SEES != RANGE) {  // row tiles of the same tokens 8 apart: on one XCD, whose L2 then reads them once
    const int each = 8 * a.row_tiles, at = blockIdx.x / each * 8 + blockIdx.x % 8;
    h = at % heads;
    r = at / heads % a.b.requests;
    split = at / heads / a.b.requests;
    rt = blockIdx.x % each / 8;
    if (split >= a.splits) return;
  }
  const Request q = request_of(a.b, r);
  const int rows = q.n * a.group, first = rt * NQ * 16;
  if (first >= rows) return;
  const int last = min(rows, first + NQ * 16) - 1;

  // tokens that any of the tile's rows sees, in tiles of 64
  Reach rf = reach_of(a, q, first / a.group), rl = reach_of(a, q, last / a.group);
  Canopy cp{};
  if constexpr (SEES == TREE) {
    cp = canopy_of(a, q, r);
    rf = {cp.low, cp.context};
    rl = {cp.high, cp.end};
  }
  const int lo = rf.lo, hi = rl.hi;
  const Tiles<SEES> tiles(a, lo, hi);
  const int tile0 = tiles.first, ntiles = tiles.count;
  const int per = SEES == RANGE ? (ntiles + a.splits - 1) / a.splits : a.chunk;
  if (SEES != RANGE && split > 0 && split * per >= ntiles) return;  // (the join knows)
  const int tb = tile0 + min(ntiles, split * per), te = tile0 + min(ntiles, (split + 1) * per);

  const int32_t *table = a.b.table + (int64_t)r * a.b.max_pages;
  const int kc = (col >> 2) * 16, vc = c * 16;  // first tokens of the chunks this lane loads
  auto entry = [&](int tok) __attribute__((always_inline)) { return table[(uint32_t)min(tok, hi - 1) >> cv.shift]; };
  int kpage = 0, vpage = 0;
  if constexpr (SEES != RANGE) {  // (with the rows and the masks: one way to memory less)
    if (tb + wave < te) {
      kpage = entry(tiles.at(tb + wave) * 64 + kc);
      vpage = entry(tiles.at(tb + wave) * 64 + vc);
    }
  }
  // the rows' elements are on their way while the tokens' pages are looked up
  v4i raw[NQ][KS];
  int rlo[NQ], rhi[NQ];
  const uint64_t *mask[SEES == TREE ? NQ : 1];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = first + n * 16 + col;
    const bool live = row < rows;
    const int t = live ? row / a.group : 0, g = live ? row - t * a.group : 0;
    const Reach s = reach_of(a, q, t);
    rlo[n] = s.lo;
    rhi[n] = live ? s.hi : 0;
    if constexpr (SEES == TREE) mask[n] = live ? a.tree.mask + (q.row0 + t) * a.tree.words : nullptr;
    // this lane's channels of row lane % 16 (of the first row past the last): of every
    // 64 (32 where 64 do not divide the head) the 16 (8) from 16 c (8 c) on, as the keys'
    const uint16_t *p = a.q + (q.row0 + t) * a.q_row + (int64_t)(h * a.group + g) * a.q_head + c * CH;
#pragma unroll
    for (int s = 0; s < KS; ++s) raw[n][s] = load_any(p + s * 8 / CH * 4 * CH + s * 8 % CH);
  }
  if constexpr (SEES == TREE) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int row = first + n * 16 + col, t = row < rows ? row / a.group : 0;
      const Reach s = branch_of(a, q, cp, r, t);
      rlo[n] = s.lo;
      rhi[n] = row < rows ? s.hi : 0;
    }
  }
  v4f O[NQ][DT];
  float M[NQ], L[NQ];
  Unit unit;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    M[n] = -INFINITY;
    L[n] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) O[n][d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int pm = cv.page - 1;
  // The tile's operands one tile ahead: keys as soon as the scores have taken the
  // present ones, values after the second product, table entries (checked where
  // they are used: a branch on them would wait for every load in flight) one
  // tile before that.
  bool vthere = false;
  float ks = 0.0f, vs = 0.0f;
  uint32_t kx[4][D / 16];
  v4i vx[DT];
  auto load_k = [&](int tile) __attribute__((always_inline)) {
    const int kt = tiles.at(tile) * 64 + kc, vt = tiles.at(tile) * 64 + vc;
    const bool kok = ((uint32_t)kpage < (uint32_t)cv.pages) & (kt < hi);
    vthere = ((uint32_t)vpage < (uint32_t)cv.pages) & (vt < hi) & ((vt + 16 > lo) | (SEES != RANGE && vt < a.sinks));
    const int8_t *kb = cv.k + (((int64_t)(kok ? kpage : 0) * heads + h) * cv.page + (kt & pm) + (col & 3)) * D + c * CH;
    const int64_t sc = (int64_t)(vthere ? vpage : 0) * heads + h;
    ks = cv.ks[sc];
    vs = cv.vs[sc];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (CH == 16) {  // (four lanes then share 64 bytes of a row: half the cache accesses of 16 D / 4 apart)
#pragma unroll
        for (int w = 0; w < D / 64; ++w) {
          const v4i x = *(const v4i *)(kb + j * 4 * D + w * 64);
#pragma unroll
          for (int i = 0; i < 4; ++i) kx[j][4 * w + i] = (uint32_t)x[i];
        }
      } else {
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          const v2i x = *(const v2i *)(kb + j * 4 * D + w * 32);
          kx[j][2 * w] = (uint32_t)x[0];
          kx[j][2 * w + 1] = (uint32_t)x[1];
        }
      }
    }
  };
  // the next values, and the table entries of the tile after: loads end in order and
  // the next keys wait for the entries, so these come first (into the registers that
  // the values' address has just left)
  auto load_v = [&](int tile) __attribute__((always_inline)) {
    const int vt = tiles.at(tile) * 64 + vc;
    const bool ok = ((uint32_t)vpage < (uint32_t)cv.pages) & (vt < hi);
    const int8_t *vb = cv.v + (((int64_t)(ok ? vpage : 0) * heads + h) * D + col) * cv.page + (vt & pm);
    kpage = entry(tiles.at(tile + W) * 64 + kc);
    vpage = entry(tiles.at(tile + W) * 64 + vc);
#pragma unroll
    for (int d = 0; d < DT; ++d) vx[d] = *(const v4i *)(vb + d * 16 * cv.page);
  };
  if (tb + wave < te) {
    if constexpr (SEES == RANGE) {
      kpage = entry(tiles.at(tb + wave) * 64 + kc);
      vpage = entry(tiles.at(tb + wave) * 64 + vc);
    }
    load_k(tb + wave);
    load_v(tb + wave);
  }
  h8 Q[NQ][KS];
  float f[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    uint32_t mag = largest<T, KS>(raw[n]);
    mag = max(mag, (uint32_t)__shfl_xor((int)mag, 16));
    mag = max(mag, (uint32_t)__shfl_xor((int)mag, 32));
    RowScale rs = row_scale(mag);
    if (a.scale < 0.0f) rs.in = -rs.in;  // the factor of the products stays >= 0
#pragma unroll
    for (int s = 0; s < KS; ++s) Q[n][s] = scaled<T>(raw[n][s], rs.in);
    f[n] = rs.out * kLog2e * fabsf(a.scale);
  }
  // the largest exponent of the present tile's scales
  auto most_of = [&](bool there, float vst) __attribute__((always_inline)) {
    const int ve = there ? exponent_of(vst) : kNoUnit;
    return max(max(__builtin_amdgcn_readlane(ve, 0), __builtin_amdgcn_readlane(ve, 16)),
               max(__builtin_amdgcn_readlane(ve, 32), __builtin_amdgcn_readlane(ve, 48)));
  };
  if (tb + wave < te) {  // (here the operands are still on their way)
    const int first_most = most_of(vthere, vs);
    if (first_most != kNoUnit) unit.move(first_most, first_most);
  }
  auto step = [&](int tile, auto last) __attribute__((always_inline)) {
    constexpr bool more = !decltype(last)::value;
    const int t0 = tiles.at(tile) * 64, vt = t0 + vc;
    const bool there = vthere;
    const float kst = ks, vst = vs;
    // (no scale of the tile from 2^5 on, one from 2^-4 on: the unit stays)
    float vq = __builtin_ldexpf(vst, -unit.u);
    if (__any(there & (vq >= 32.0f)) || !__any(there & (vq >= 0.0625f))) {
      const int most = most_of(there, vst), was = unit.u;
      if (unit.leaves(most)) unit.move(most, most);
      const float by = __builtin_ldexpf(1.0f, was - unit.u);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int d = 0; d < DT; ++d) O[n][d] *= by;
      vq = __builtin_ldexpf(vst, -unit.u);
    }
    const ValueScale vsc = value_scale(vq);
    const float u = vsc.u, rv = vsc.rv;
    v4f S[NQ][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int n = 0; n < NQ; ++n) S[n][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const h8 A = codes_h8(kx[j][2 * s], kx[j][2 * s + 1]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) S[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, Q[n][s], S[n][j], 0, 0, 0);
      }
    if constexpr (more) load_k(tile + W);
    h8 P[NQ][2];
    // Tokens that all rows see need no masks (columns past the last row are not stored).
    // 8 requests of 17 to 131 rows, heads of 64: 18.5 us, 21.5 with masks always.  The wider
    // builds keep them: two paths took 256 registers and scratch (heads of 128, 32 rows).
    const bool whole = (SEES != RANGE || D * NQ <= 128) && __all(there) && t0 >= rl.lo && t0 + 64 <= rf.hi;
    auto weigh = [&](int n, auto masks) __attribute__((always_inline)) {
      constexpr bool some = decltype(masks)::value;
      const float fk = f[n] * kst;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (some) {
            const int tok = vt + 4 * j + i;
            const bool sees = there & (tok >= rlo[n]) & (tok < rhi[n]);
            S[n][j][i] = sees ? __builtin_fmaf(S[n][j][i], fk, u) : -INFINITY;
          }
          mx = fmaxf(mx, S[n][j][i]);
        }
      // (fk >= 0: the largest score comes from the largest product)
      if constexpr (!some) mx = mx == -INFINITY ? -INFINITY : __builtin_fmaf(mx, fk, u);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      if (__any(mx > M[n] + kSlack)) {
        const float mn = fmaxf(M[n], mx), alpha = exp2_fast(M[n] - (mn == -INFINITY ? 0.0f : mn));
        M[n] = mn;
        L[n] *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d) O[n][d] *= alpha;
      }
      const float ms = M[n] == -INFINITY ? 0.0f : M[n], o = u - ms;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(some ? S[n][j][i] - ms : __builtin_fmaf(S[n][j][i], fk, o));
          sum += p;
          P[n][j >> 1][(j & 1) * 4 + i] = (_Float16)p;
        }
      L[n] += sum == 0.0f ? 0.0f : sum * rv;
    };
    // Sinks and trees mask the products themselves, -inf times a factor above 0 (or 1, where a chunk's
    // scales may be NaN and nothing of it is seen), so that one path without masks follows in every
    // build, all rows together.  8 drafts of 25 tokens, heads of 96 in groups of 7, window 4095: 31.3 us, 33.9 with
    // masks at every score; 16 drafts of 64, heads of 128, in blocks of 32 rows: 269, 902 (registers go to scratch).
    auto weigh_masked = [&]() __attribute__((always_inline)) {
      float fk[NQ], un[NQ], mx[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        fk[n] = f[n] * kst;
        un[n] = u;
      }
      if (!whole) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const uint32_t seen = there ? seen16(a, q, vt, rlo[n], rhi[n], cp, SEES == TREE ? mask[n] : nullptr) : 0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[n][j][i] = seen >> (4 * j + i) & 1 ? S[n][j][i] : -INFINITY;
          fk[n] = seen == 0 ? 1.0f : fk[n] == 0.0f ? 1.17549435e-38f : fk[n];
          un[n] = seen == 0 ? 0.0f : u;
        }
      }
      bool up = false;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) m = fmaxf(m, S[n][j][i]);
        m = m == -INFINITY ? -INFINITY : __builtin_fmaf(m, fk[n], un[n]);
        mx[n] = other_half_max(other_row_max(m));
        up |= mx[n] > M[n] + kSlack;
      }
      if (__any(up)) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const float mn = fmaxf(M[n], mx[n]), alpha = exp2_fast(M[n] - (mn == -INFINITY ? 0.0f : mn));
          M[n] = mn;
          L[n] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) O[n][d] *= alpha;
        }
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float o = un[n] - (M[n] == -INFINITY ? 0.0f : M[n]);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = exp2_fast(__builtin_fmaf(S[n][j][i], fk[n], o));
            sum += p;
            P[n][j >> 1][(j & 1) * 4 + i] = (_Float16)p;
          }
        L[n] += sum == 0.0f ? 0.0f : sum * rv;
      }
    };
    if constexpr (SEES != RANGE) {
      weigh_masked();
    } else if (whole) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) weigh(n, std::false_type());
    } else {
#pragma unroll
      for (int n = 0; n < NQ; ++n) weigh(n, std::true_type());
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const h8 A = codes_h8((uint32_t)vx[d][2 * s], (uint32_t)vx[d][2 * s + 1], vsc.m, vsc.n);
#pragma unroll
        for (int n = 0; n < NQ; ++n) O[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, P[n][s], O[n][d], 0, 0, 0);
      }
    if constexpr (more) load_v(tile + W);
  };
  // (the last step apart: under a condition, loads would be waited for as if there were none)
  int tile = tb + wave;
  for (; tile + W < te; tile += W) step(tile, std::false_type());
  if (tile < te) step(tile, std::true_type());

  // the waves' results under one maximum and in one unit
  if (lane == 0) su[wave] = unit.u;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float l = L[n];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (c == 0) {
      sm[wave][n * 16 + col] = M[n];
      sl[wave][n * 16 + col] = l;
    }
  }
  __syncthreads();
  int ut = max(max(su[0], su[1]), max(su[2], su[3]));
#pragma unroll
  for (int w = 4; w < W; ++w) ut = max(ut, su[w]);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int rc = n * 16 + col;
    float mt = fmaxf(fmaxf(sm[0][rc], sm[1][rc]), fmaxf(sm[2][rc], sm[3][rc]));
#pragma unroll
    for (int w = 4; w < W; ++w) mt = fmaxf(mt, sm[w][rc]);
    const float wgt = __builtin_ldexpf(exp2_fast(M[n] - (mt == -INFINITY ? 0.0f : mt)), unit.u - ut);
#pragma unroll
    for (int d = 0; d < DT; ++d) *(v4f *)&so[wave][col * OLD + d * 16 + c * 4] = O[n][d] * wgt;
    __syncthreads();
    for (int p = threadIdx.x; p < 16 * (D / 4); p += 64 * W) {
      const int qr = p / (D / 4), d = p % (D / 4) * 4, row = first + n * 16 + qr;
      if (row >= rows) continue;
      const int t = row / a.group, hq = h * a.group + row - t * a.group;
      v4f o = *(v4f *)&so[0][qr * OLD + d];
#pragma unroll
      for (int w = 1; w < W; ++w) o += *(v4f *)&so[w][qr * OLD + d];
      const int rq = n * 16 + qr;
      float m = -INFINITY, l = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) m = fmaxf(m, sm[w][rq]);
#pragma unroll
      for (int w = 0; w < W; ++w) l += sl[w][rq] * exp2_fast(sm[w][rq] - (m == -INFINITY ? 0.0f : m));
      if (a.splits == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const float v[4] = {__builtin_ldexpf(o[0] * inv, ut), __builtin_ldexpf(o[1] * inv, ut), __builtin_ldexpf(o[2] * inv, ut),
                            __builtin_ldexpf(o[3] * inv, ut)};
        uint16_t *dst = a.out + (q.row0 + t) * a.out_row + (int64_t)hq * a.out_head + d;
        store4<T>(dst, v);
      } else {
        const int64_t hs = (int64_t)cv.heads * a.group;
        const int64_t at = ((int64_t)split * a.b.tokens + q.row0 + t) * hs + hq;
        *(v4f *)(a.part + at * D + d) = o;
        if (d == 0) *(v4f *)(a.part + (int64_t)a.splits * a.b.tokens * hs * D + at * 4) = v4f{m, l, (float)ut, 0.0f};
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------ many rows
// Prompts: a workgroup of 4 waves takes 128 (query, head) rows of one cache head, a
// wave 32 of them on v_mfma_f32_32x32x16_f16, in the layout above (a lane has one query
// and, of every 32 tokens, 16 consecutive ones).  The workgroup's 64-token tiles are read
// as codes a tile ahead, converted to fp16 once and kept in LDS for all waves, one
// barrier a tile; two workgroups on a CU (up to 128 channels) fill each other's gaps.
// 4 requests, 1531 to 2048 tokens behind cached ones, 2100 to 4096 in all, 8 heads of
// 128, group 4: 324 us, 766 TFLOP/s (a bf16 library product of 8192^3: 1240 to 1270).  A
// wave's step of 64 tokens takes about 4000 cycles alone, 1024 of them products; the softmax
// is 28 % of the time (232 us without), the conversion 9 % (294).
//
// LDS holds each matrix operand as the 1 KB that a wave reads, lane after lane, so
// a read is a lane's own address plus a constant and meets no bank twice; the
// threads that bring a tile are arranged so that 8 neighbours write 8 neighbouring
// lanes' pieces (row 8 g + 4 c + i of a subtile of keys is token 16 c + 4 g + i).
//

template <int D>
struct TileLds {
  static constexpr int KEYS = 64 * D * 2;            // bytes of a tile's keys, and of its values
  static constexpr int OUT = 128 * (D * 2 + 16);  // the epilogue's rows
  static constexpr int BYTES = 4 * KEYS > OUT ? 4 * KEYS : OUT;
};

// Keeps kAhead operand reads in flight before the N products of this block: an LDS
// read takes the time of four products, and the compiler by itself asks for one
// operand at a time (4 requests, 2048 tokens of 4096: 450 us, 457 without).  With one more in
// flight the narrow pages' build for heads of 128 has no registers left for any: 153 us become
// 167 (4 requests, 900 to 1100 tokens of 2048, pages of 32).
constexpr int kAhead = 4;
template <int N>
__device__ __forceinline__ void ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);  // LDS reads
#pragma unroll
  for (int j = 0; j < N - kAhead; ++j) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix product
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
}

template <class T, int D, bool WIDE, int SEES>
__global__ __launch_bounds__(256, D > 128 ? 1 : 2) void attend_tile_kernel(AttendArgs a, int first_tile, int row_tiles) {
  typedef TileLds<D> G;
  constexpr int ROWS = 128, KS = D / 16, DT = D / 32, PP = (4 * D + kTileThreads - 1) / kTileThreads;
  __shared__ __attribute__((aligned(256))) uint8_t lds[G::BYTES];
  __shared__ float4 blocks[4][4];  // of four tiles' 16-token chunks: {ks, u, 1 / r, page there}
  __shared__ uint32_t factors[4][4];  // narrow pages: and the factor of their values' codes
  __shared__ int units[4];            // and the tiles' units
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, c = lane >> 5;
  // cache heads go fastest, so a head's tiles share one XCD's L2 where heads are a
  // multiple of 8; the rows with the longest reach start first
  const int heads = a.c.heads, combos = heads * a.b.requests;
  const int combo = blockIdx.x % combos, rest = blockIdx.x / combos;
  const int h = combo % heads, r = (combo / heads + rest) % a.b.requests, split = rest % a.splits, rt = first_tile + row_tiles - 1 - rest / a.splits;
  const CacheView &cv = a.c;
  const Request q = request_of(a.b, r);
  const int rows = q.n * a.group, first = rt * ROWS;
  if (first >= rows) return;
  const int last = min(rows, first + ROWS) - 1;
  Reach rf = reach_of(a, q, first / a.group), rl = reach_of(a, q, last / a.group);
  Canopy cp{};
  if constexpr (SEES == TREE) {
    cp = canopy_of(a, q, r);
    rf = {cp.low, cp.context};
    rl = {cp.high, cp.end};
  }
  const int hi = rl.hi;
  const Tiles<SEES> tiles(a, rf.lo, hi);
  const int tile0 = tiles.first, ntiles = tiles.count;
  const int per = SEES == RANGE ? (ntiles + a.splits - 1) / a.splits : a.chunk;
  if (SEES != RANGE && split > 0 && split * per >= ntiles) return;  // (the join knows)
  const int tb = tile0 + min(ntiles, split * per), te = tile0 + min(ntiles, (split + 1) * per);

  // this wave's rows
  const int row = first + wave * 32 + col;
  const bool live = row < rows;
  const int t = live ? row / a.group : 0, hq = h * a.group + (live ? row - t * a.group : 0);
  const Reach mine = SEES == TREE ? branch_of(a, q, cp, r, t) : reach_of(a, q, t);
  const int rlo = mine.lo, rhi = live ? mine.hi : 0;
  const uint64_t *mask = SEES == TREE && live ? a.tree.mask + (q.row0 + t) * a.tree.words : nullptr;
  // tokens that all of the wave's rows see, and that any sees
  const int w0 = first + wave * 32, w1 = min(w0 + 31, last);
  const Reach wf = SEES == TREE ? rf : reach_of(a, q, min(w0, last) / a.group), wl = SEES == TREE ? rl : reach_of(a, q, w1 / a.group);
  const int all_lo = wl.lo, all_hi = w0 + 31 <= last ? wf.hi : 0, any_lo = wf.lo, any_hi = w0 <= last ? wl.hi : 0;

  h8 Q[KS];
  float f;
  {
      const uint16_t *p = a.q + (q.row0 + t) * a.q_row + (int64_t)hq * a.q_head + c * 8;
    v4i raw[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) raw[s] = load_any(p + s * 16);
    uint32_t mag = largest<T, KS>(raw);
    mag = max(mag, (uint32_t)__shfl_xor((int)mag, 32));
    RowScale rs = row_scale(mag);
    if (a.scale < 0.0f) rs.in = -rs.in;  // the factor of the products stays >= 0
#pragma unroll
    for (int s = 0; s < KS; ++s) Q[s] = scaled<T>(raw[s], rs.in);
    f = rs.out * kLog2e * fabsf(a.scale);
  }

  const int32_t *table = a.b.table + (int64_t)r * a.b.max_pages;
  const int pm = cv.page - 1;
  // table entry of a token's page (of the last token's past it), checked only where
  // it is used: a branch on it here would wait for every load in flight
  auto entry = [&](int tok) __attribute__((always_inline)) { return table[(uint32_t)min(tok, hi - 1) >> cv.shift]; };
  auto valid = [&](int pid) __attribute__((always_inline)) { return (uint32_t)pid < (uint32_t)cv.pages; };
  // The 16-byte pieces that this thread brings: 16 channels of a key of tile p and 16
  // tokens of a value channel of tile p - 1.
  auto piece = [&](int i) __attribute__((always_inline)) { return tile_piece((int)threadIdx.x + i * kTileThreads, D); };
  auto none = [&](int i) __attribute__((always_inline)) { return tile_piece_past((int)threadIdx.x + i * kTileThreads, D); };
  // Table entries go through two sets of registers by the tile's parity (a copy from
  // one to the other would wait for them, and so for every load before them).
  // WIDE (pages of a tile or more): the entries are the same for all threads and stay in
  // scalar registers, as do the pages' addresses.
  // With sinks or trees narrow pages' entries do, too, where heads have 64 or 256 channels: four chunks' of a
  // tile, its values' kept from its keys', and a thread selects its pieces' pages.  That takes vector instructions and
  // registers for scalar ones: 4 prompts, window 1024, pages of 32: 141 us against 161 for heads of 64, 665 against 737
  // for 256, but 223 against 216 for 128 and 216 against 190 for 96.
  constexpr bool CHUNKS = !WIDE && SEES != RANGE && (D == 64 || D == 256);
  struct Entries { int k[WIDE ? 1 : CHUNKS ? 4 : PP], v[WIDE || CHUNKS ? 1 : PP], b; } ent[2];
  int vpages[CHUNKS ? 4 : 1];
  v4i kx[PP], vx[PP];
  float bks, bvs, bthere;  // of chunk threadIdx.x % 4 of tile p
  const uint32_t page_bytes = (uint32_t)heads << cv.shift;  // (times D)
  const int8_t *kh = cv.k + ((int64_t)h << cv.shift) * D, *vh = cv.v + ((int64_t)h << cv.shift) * D;
  typedef const __attribute__((address_space(4))) int32_t *ScalarInts;
  typedef const __attribute__((address_space(4))) float *ScalarFloats;
  auto entries = [&](int p, Entries &e) __attribute__((always_inline)) {
    if constexpr (WIDE) {
      const ScalarInts st = (ScalarInts)(uintptr_t)table;
      e.k[0] = e.b = st[__builtin_amdgcn_readfirstlane((uint32_t)min(tiles.at(p) * 64, hi - 1) >> cv.shift)];
      e.v[0] = st[__builtin_amdgcn_readfirstlane((uint32_t)min(tiles.at(max(p - 1, tb)) * 64, hi - 1) >> cv.shift)];
      return;
    }
    if constexpr (CHUNKS) {
      const ScalarInts st = (ScalarInts)(uintptr_t)table;
#pragma unroll
      for (int j = 0; j < 4; ++j) e.k[j] = st[__builtin_amdgcn_readfirstlane((uint32_t)min(tiles.at(p) * 64 + j * 16, hi - 1) >> cv.shift)];
      return;
    }
#pragma unroll
    for (int i = 0; i < PP; ++i) {
      e.k[i] = entry(tiles.at(p) * 64 + piece(i).tok);
      e.v[i] = entry(tiles.at(max(p - 1, tb)) * 64 + piece(i).vt);
    }
    e.b = entry(tiles.at(p) * 64 + (threadIdx.x & 3) * 16);
  };
  auto load = [&](int p, const Entries &e) __attribute__((always_inline)) {
    const int ktile = tiles.at(p) * 64 & pm, vtile = tiles.at(max(p - 1, tb)) * 64 & pm;  // of a page that is wider than a tile
    if constexpr (WIDE) {
      const int kp = __builtin_amdgcn_readfirstlane(valid(e.k[0]) ? e.k[0] : 0), vp = __builtin_amdgcn_readfirstlane(valid(e.v[0]) ? e.v[0] : 0);
      const int8_t *kt = kh + (uint64_t)kp * page_bytes * D, *vt = vh + (uint64_t)vp * page_bytes * D;
#pragma unroll
      for (int i = 0; i < PP; ++i) {
        const TilePiece pc = piece(i);
        kx[i] = *(const v4i *)(kt + tile_key_at(pc, ktile, 63, D));
        vx[i] = *(const v4i *)(vt + tile_value_at(pc, vtile, 63, cv.shift));
      }
      const int64_t at = (int64_t)kp * heads + h;
      bks = ((ScalarFloats)(uintptr_t)cv.ks)[at];
      bvs = ((ScalarFloats)(uintptr_t)cv.vs)[at];
      bthere = valid(e.b) ? 1.0f : 0.0f;
      return;
    }
    if constexpr (CHUNKS) {
      // the start of the page that holds 16 tokens from chunk 16 on
      auto page_of = [&](const int *ids, const int8_t *base, int chunk) __attribute__((always_inline)) {
        uint64_t at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) at[j] = (uint64_t)base + (uint64_t)(uint32_t)(valid(ids[j]) ? ids[j] : 0) * page_bytes * D;
        const uint64_t even = chunk & 2 ? at[2] : at[0], odd = chunk & 2 ? at[3] : at[1];
        return (const int8_t *)(chunk & 1 ? odd : even);
      };
      const int8_t *vp = page_of(vpages, vh, piece(0).vt >> 4);  // (a thread's pieces are 256 apart: the same tokens)
#pragma unroll
      for (int i = 0; i < PP; ++i) {
        const TilePiece pc = piece(i);
        kx[i] = *(const v4i *)(page_of(e.k, kh, pc.tok >> 4) + tile_key_at(pc, ktile, pm, D));
        vx[i] = *(const v4i *)(vp + tile_value_at(pc, vtile, pm, cv.shift));
      }
      const int c4 = threadIdx.x & 3, even = c4 & 2 ? e.k[2] : e.k[0], odd = c4 & 2 ? e.k[3] : e.k[1], id = c4 & 1 ? odd : even;
      const int chunk = tiles.at(p) * 64 + c4 * 16;  // (what no row sees sets no unit)
      const int64_t at = (int64_t)(valid(id) ? id : 0) * heads + h;
      bks = cv.ks[at];
      bvs = cv.vs[at];
      bthere = valid(id) && (chunk + 16 > rf.lo || chunk < a.sinks) ? 1.0f : 0.0f;
      return;
    }
#pragma unroll
    for (int i = 0; i < PP; ++i) {
      const TilePiece pc = piece(i);
      const uint64_t kp = (uint64_t)(uint32_t)(valid(e.k[i]) ? e.k[i] : 0) * page_bytes * D;
      const uint64_t vp = (uint64_t)(uint32_t)(valid(e.v[i]) ? e.v[i] : 0) * page_bytes * D;
      kx[i] = *(const v4i *)(kh + kp + tile_key_at(pc, ktile, pm, D));
      vx[i] = *(const v4i *)(vh + vp + tile_value_at(pc, vtile, pm, cv.shift));
    }
    const bool page = valid(e.b);
    const int chunk = tiles.at(p) * 64 + (int)(threadIdx.x & 3) * 16;  // (what no row sees sets no unit)
    const bool reached = (chunk + 16 > rf.lo) | (SEES != RANGE && chunk < a.sinks);
    const int64_t at = (int64_t)(page ? e.b : 0) * heads + h;
    bks = cv.ks[at];
    bvs = cv.vs[at];
    bthere = page && reached ? 1.0f : 0.0f;
  };
  // keys of tile p and values of tile p - 1 to their places, then the loads of the
  // next.  Loads end in order, so the entries that the next call needs come first.
  // None of it stands under a condition, so that waits count only what they need; past
  // the last tile it reads tiles that nobody uses.  par: p - tb is odd.
  // The units of two tiles, by their parity, in scalar registers.  WIDE: one scale a tile,
  // which every wave follows; else wave 0 follows the four chunks', and the others read LDS
  // after a step's barrier for the next step, with the factor of this thread's 16 tokens.
  Unit unit;
  int tile_unit[2] = {kNoUnit, kNoUnit}, next_unit = kNoUnit;
  uint32_t factor = 0;
  auto see_blocks = [&](int p) __attribute__((always_inline)) {
    if constexpr (!WIDE) {
      next_unit = units[(p - tb) & 3];
      factor = factors[(p - tb) & 3][threadIdx.x >> 4 & 3];  // (a thread's pieces are 256 apart: the same tokens)
    }
  };
  auto bring_blocks = [&](int p, auto par) __attribute__((always_inline)) {
    if constexpr (WIDE) {
      const int e = valid(ent[decltype(par)::value].b) ? exponent_of(bvs) : kNoUnit;
      if (e != kNoUnit && (e < unit.u || e > unit.u + 4)) unit.move(e - 2, e);
      tile_unit[decltype(par)::value] = unit.u;
      if (wave == 0 && lane < 4) {
        const ValueScale v = value_scale(__builtin_ldexpf(bvs, -unit.u), true);
        blocks[(p - tb) & 3][lane] = make_float4(bks, v.u, v.rv, bthere);
      }
    } else if (wave == 0) {
      const int e = bthere != 0.0f ? exponent_of(bvs) : kNoUnit;
      int most = max(e, __builtin_amdgcn_mov_dpp(e, 0xB1, 0xf, 0xf, true));  // of the lane's four, which are the tile's
      most = __builtin_amdgcn_readfirstlane(max(most, __builtin_amdgcn_mov_dpp(most, 0x4E, 0xf, 0xf, true)));
      if (unit.leaves(most)) unit.move(most, most);
      const ValueScale v = value_scale(__builtin_ldexpf(bvs, -unit.u));
      if (lane < 4) {
        blocks[(p - tb) & 3][lane] = make_float4(bks, v.u, v.rv, bthere);
        factors[(p - tb) & 3][lane] = v.m;
      }
      if (lane == 0) units[(p - tb) & 3] = unit.u;
    }
  };
  auto bring = [&](int p, auto par) __attribute__((always_inline)) {
    constexpr int odd = decltype(par)::value;
    uint8_t *kbase = lds + odd * G::KEYS, *vbase = lds + (2 + (odd ^ 1)) * G::KEYS;
    const uint32_t less = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, factor) * h2{(_Float16)-1152.0f, (_Float16)-1152.0f});
#pragma unroll
    for (int i = 0; i < PP; ++i) {
      if (none(i)) break;
      const TilePiece pc = piece(i);
      // operand (subtile, 16 channels): lane 32 c + row has 8 channels from 8 c
      uint8_t *kd = kbase + ((pc.kr >> 5) * KS + pc.s) * 1024 + (pc.kr & 31) * 16;
      *(h8 *)kd = codes_h8((uint32_t)kx[i][0], (uint32_t)kx[i][1]);
      *(h8 *)(kd + 512) = codes_h8((uint32_t)kx[i][2], (uint32_t)kx[i][3]);
      // operand (32 channels, subtile, k): lane 32 c + channel has 8 tokens from 16 c + 8 k
      uint8_t *vd = vbase + (pc.d >> 5) * 4096 + (pc.vt >> 5) * 2048 + (pc.vt >> 4 & 1) * 512 + (pc.d & 31) * 16;
      if constexpr (WIDE) {
        *(h8 *)vd = codes_h8((uint32_t)vx[i][0], (uint32_t)vx[i][1]);
        *(h8 *)(vd + 1024) = codes_h8((uint32_t)vx[i][2], (uint32_t)vx[i][3]);
      } else {
        *(h8 *)vd = codes_h8((uint32_t)vx[i][0], (uint32_t)vx[i][1], factor, less);
        *(h8 *)(vd + 1024) = codes_h8((uint32_t)vx[i][2], (uint32_t)vx[i][3], factor, less);
      }
    }
    if constexpr (CHUNKS)
#pragma unroll
      for (int j = 0; j < 4; ++j) vpages[j] = ent[odd].k[j];
    entries(p + 2, ent[odd]);
    load(p + 1, ent[odd ^ 1]);
  };

  v16f O[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[d][i] = 0.0f;
  float M = -INFINITY, L = 0.0f;
  int ou = kNoUnit;  // the unit of O
  v16f S[2];
  h8 P[2][2];
  bool busy = false;  // this wave has scores, or weights, of the present tile
  const uint8_t *mylds = lds + lane * 16;

  auto second = [&](auto which) __attribute__((always_inline)) {  // of the tile before one of this parity
    constexpr int b = decltype(which)::value;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const h8 *)(mylds + (2 + (b ^ 1)) * G::KEYS + d * 4096 + k * 1024),
                                                       P[k >> 1][k & 1], O[d], 0, 0, 0);
    ahead<4 * DT>();
  };
  auto scores = [&](auto which) __attribute__((always_inline)) {  // of a tile of this parity
    constexpr int b = decltype(which)::value;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) S[u][j] = 0.0f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        S[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const h8 *)(mylds + b * G::KEYS + (u * KS + s) * 1024), Q[s], S[u], 0, 0, 0);
    ahead<2 * KS>();
  };
  // matrix phase of tile i: the next tile's way to LDS, the second product of tile i - 1,
  // the first of tile i
  auto products = [&](int i, auto which) __attribute__((always_inline)) {
    constexpr std::integral_constant<int, decltype(which)::value ^ 1> other;
    const int t0 = tiles.at(i) * 64;
    const bool next = i < te && t0 < any_hi && (t0 + 64 > any_lo || (SEES != RANGE && t0 < a.sinks));
    if (i < te) {
      if constexpr (!WIDE) tile_unit[decltype(which)::value] = __builtin_amdgcn_readfirstlane(next_unit);
      bring_blocks(i + 1, other);
      bring(i + 1, other);
    }
    if (busy) second(which);
    if (next) scores(which);
    busy = next;
  };
  // vector phase: the weights of tile i
  auto weigh = [&](int i, auto which) __attribute__((always_inline)) {
    constexpr int b = decltype(which)::value;
    if (!busy) return;
    const int t0 = tiles.at(i) * 64;
    const float4 b0 = blocks[(i - tb) & 3][c], b1 = blocks[(i - tb) & 3][2 + c];
    const int moved = ou - tile_unit[b];
    ou = tile_unit[b];
    if (D <= 128 && moved) {
      const float by = __builtin_ldexpf(1.0f, moved);
#pragma unroll
      for (int d = 0; d < DT; ++d) O[d] *= by;
    }
    // tokens of this lane that its row does not see, where there are any
    const bool masked = !(__all(b0.w != 0.0f && b1.w != 0.0f) && t0 >= all_lo && t0 + 64 <= all_hi);
    uint32_t off = 0;
    if (masked) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bool ok = (u ? b1.w : b0.w) != 0.0f;
        if constexpr (SEES != RANGE) off |= (ok ? ~seen16(a, q, t0 + u * 32 + c * 16, rlo, rhi, cp, mask) & 0xffffu : 0xffffu) << (u * 16);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int tok = t0 + u * 32 + c * 16 + j;
          const bool sees = SEES == RANGE ? ok & (tok >= rlo) & (tok < rhi) : !(off >> (u * 16 + j) & 1u);
          if constexpr (SEES == RANGE) off |= sees ? 0u : 1u << (u * 16 + j);
          S[u][j] = sees ? S[u][j] : -INFINITY;
        }
      }
    }
    // s fk + lv, fk >= 0: the largest comes from the largest product.  Of lv only the fraction, so that a
    // wide tile's whole powers of two (up to 4) take nothing from the others, and the largest weight is a
    // power of two, which fp16 holds exactly: rows with few tokens gain most.
    float fk[2] = {f * b0.x, f * b1.x}, lv[2] = {b0.y, b1.y};
    if (SEES != RANGE && masked)  // (as in attend_rows_kernel: -inf times a factor above 0 needs no second mask)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bool none = (off >> (u * 16) & 0xffffu) == 0xffffu;
        fk[u] = none ? 1.0f : fk[u] == 0.0f ? 1.17549435e-38f : fk[u];
        lv[u] = none ? 0.0f : lv[u];
      }
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < 16; ++j) m = fmaxf(m, S[u][j]);
      mx = fmaxf(mx, m == -INFINITY ? -INFINITY : __builtin_fmaf(m, fk[u], __builtin_amdgcn_fractf(lv[u])));
    }
    mx = other_half_max(mx);
    // (heads of 256: one place for both, a second costs 6 %; smaller ones: two, 0.5 %)
    if ((D > 128 && moved) || __any(mx > M + kSlack)) {
      const float mn = fmaxf(M, mx), alpha = exp2_fast(M - (mn == -INFINITY ? 0.0f : mn));
      const float by = D > 128 ? __builtin_ldexpf(alpha, moved) : alpha;
      M = mn;
      L *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) O[d] *= by;
    }
    const float ms = M == -INFINITY ? 0.0f : M;
    auto weights = [&](auto some) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float o = lv[u] - ms;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          float p = exp2_fast(__builtin_fmaf(S[u][j], fk[u], o));
          if constexpr (decltype(some)::value) p = off >> (u * 16 + j) & 1u ? 0.0f : p;
          sum += p;
          P[u][j >> 3][j & 7] = (_Float16)p;
        }
        L += sum == 0.0f ? 0.0f : sum * (u ? b1.z : b0.z);
      }
    };
    if (SEES == RANGE && masked) weights(std::true_type());
    else weights(std::false_type());
  };

  if (tb < te) {
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    entries(tb, ent[0]);
    entries(tb + 1, ent[1]);
    if constexpr (CHUNKS)
#pragma unroll
      for (int j = 0; j < 4; ++j) vpages[j] = ent[0].k[j];
    load(tb, ent[0]);
    bring_blocks(tb, even);
    bring(tb, even);  // (there are no values yet: those of tile tb, twice)
    __syncthreads();
    see_blocks(tb);
    // One barrier a step: what a step brings to LDS is read in the next, and takes the
    // place of what was read in the step before.
    auto both = [&](int i, auto which) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);  // before the CU's other workgroup in its softmax
      products(i, which);
      __builtin_amdgcn_s_setprio(0);
      __syncthreads();
      see_blocks(i + 1);
      if (i < te) weigh(i, which);
    };
    for (int i = tb; i <= te; i += 2) {
      both(i, even);
      if (i + 1 <= te) both(i + 1, odd);
    }
  }
  __syncthreads();

  L += __shfl_xor(L, 32);
  if (a.splits > 1) {
    if (!live) return;
    const int64_t hs = (int64_t)heads * a.group, at = ((int64_t)split * a.b.tokens + q.row0 + t) * hs + hq;
    float *dst = a.part + at * D;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(v4f *)(dst + d * 32 + g * 8 + c * 4) = v4f{O[d][4 * g], O[d][4 * g + 1], O[d][4 * g + 2], O[d][4 * g + 3]};
    if (c == 0) *(v4f *)(a.part + (int64_t)a.splits * a.b.tokens * hs * D + at * 4) = v4f{M, L, (float)ou, 0.0f};
    return;
  }
  // rows through LDS (the last barrier came after every wave's last read), a wave's own part
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  constexpr int LD = D + 8;
  uint16_t *my = (uint16_t *)lds + wave * 32 * LD;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __builtin_ldexpf(O[d][4 * g + i] * inv, ou);
      store4<T>(my + col * LD + d * 32 + g * 8 + c * 4, v);
    }
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  for (int p = lane; p < 32 * (D / 8); p += 64) {
    const int rr = p / (D / 8), e = p % (D / 8) * 8, orow = first + wave * 32 + rr;
    if (orow >= rows) continue;
    const int ot = orow / a.group, oh = h * a.group + orow - ot * a.group;
    const v4i o = *(const v4i *)(my + rr * LD + e);
    uint16_t *dst = a.out + (q.row0 + ot) * a.out_row + (int64_t)oh * a.out_head + e;
    store_any(dst, o);
  }
}

// One (token, head) row a group of D / 4 threads: the splits under one maximum and
// in one unit.
template <class T, int D, int SEES>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int W = D / 4;
  const int r = blockIdx.y;
  const Request q = request_of(a.b, r);
  const int hs = a.c.heads * a.group, sub = threadIdx.x / W, d = threadIdx.x % W * 4;
  const int64_t i = (int64_t)blockIdx.x * (256 / W) + sub;
  if (sub >= 256 / W || i >= (int64_t)q.n * hs) return;
  const int64_t t = i / hs, hq = i - t * hs, at = (q.row0 + t) * hs + hq, step = a.b.tokens * hs;
  const float *ml = a.part + a.splits * step * D;
  int splits = a.splits;
  if constexpr (SEES != RANGE) {  // the parts that the row's block has
    const int row = (int)t * a.group + (int)hq % a.group, first = row / a.block * a.block, last = min(q.n * a.group, first + a.block) - 1;
    int lo, hi;
    if constexpr (SEES == TREE) {
      const Canopy cp = canopy_of(a, q, r);
      lo = cp.low;
      hi = cp.end;
    } else {
      lo = reach_of(a, q, first / a.group).lo;
      hi = reach_of(a, q, last / a.group).hi;
    }
    splits = max(1, min(splits, (Tiles<SEES>(a, lo, hi).count + a.chunk - 1) / a.chunk));
  }
  // eight splits at a time, all their loads in flight
  float m = -INFINITY, l = 0.0f, u = kNoUnit;
  v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < splits; s0 += 8) {
    v4f x[8];
    v4f y[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int64_t from = min(s0 + s, splits - 1) * step + at;
      x[s] = *(const v4f *)(ml + from * 4);
      y[s] = *(const v4f *)(a.part + from * D + d);
    }
    float mn = m, un = u;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      mn = fmaxf(mn, x[s][0]);
      un = fmaxf(un, x[s][2]);
    }
    const float ms = mn == -INFINITY ? 0.0f : mn, w0 = exp2_fast(m - ms);
    l *= w0;
    o *= __builtin_ldexpf(w0, (int)(u - un));
    m = mn;
    u = un;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const float w = s0 + s < splits ? exp2_fast(x[s][0] - ms) : 0.0f;
      l += x[s][1] * w;
      o += y[s] * __builtin_ldexpf(w, (int)(x[s][2] - u));
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  float v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = __builtin_ldexpf(o[k] * inv, (int)u);
  uint16_t *dst = a.out + (q.row0 + t) * a.out_row + hq * a.out_head + d;
  store4<T>(dst, v);
}

// Waves of attend_rows_kernel's workgroups: eight with sinks or trees, whose rows then need fewer parts that
// are joined through memory (one token of a window of 512: 6.8 us, 7.4 with four; 32 of a window of 4096: 50.1, 51.2; 8
// drafts of 25: 31.4, 35.3); heads of 256 have registers for four.
constexpr int rows_waves(int dim, int sees) { return sees != RANGE && dim < 256 ? 8 : 4; }

// Tokens that a request has rows for at most.  (max_new itself counts from the request's start, which may lie before the
// first row.)
int64_t most_new(const AttendArgs &a) { return std::min<int64_t>(a.b.max_new, a.b.tokens); }

// Rows of a workgroup: 16 or 32 on attend_rows_kernel, 128 on attend_tile_kernel.
// While the small blocks are at most 3 for each CU, their many waves over the
// tokens end sooner than the tile kernel's long chain of steps, although each
// block converts its codes itself: 4 requests, 8 heads, group 4, 2048 tokens, 64 /
// 128 / 256 new ones: 29 / 39 / 72 us against 35 / 40 / 58.  Drafts whose rows fill
// blocks of 128 go there from one small block for each CU on if they are behind 8192 tokens
// or more (4 / 8 / 12 drafts of 64 behind 8000 to 16000: 88 / 176 / 256 us, 104 / 184 / 280 in small
// blocks; behind 1000 to 2000 61 / 64 / 64, 23 / 42 / 63).
int block_rows(const AttendArgs &a, int cus) {
  const int64_t rows = most_new(a) * a.group, small = rows <= 16 || a.c.dim == 256 ? 16 : 32;
  const int64_t blocks = (rows + small - 1) / small * a.c.heads * a.b.requests;
  if (a.tree.mask && a.window == 0 && a.b.max_len >= 8192 && (rows + 127) / 128 * 128 * 8 <= rows * 9 && blocks >= cus) return 128;
  return blocks <= 3 * cus ? (int)small : 128;
}

template <class T, int D, int SEES>
hipError_t launch_attend_d(const AttendArgs &a, hipStream_t s) {
  const int64_t rows = most_new(a) * a.group, rt = (rows + a.block - 1) / a.block;
  if (a.block == 128) {
    // one launch, unless loose bounds make it too large: then the last rows' first
    const int64_t each = (int64_t)a.splits * a.c.heads * a.b.requests, most = kMaxGroups / each;
    for (int64_t left = rt; left > 0; left -= most) {
      const int64_t n = std::min(left, most), t0 = left - n;
      const unsigned flat = (unsigned)(n * each);
      if (a.c.page >= 64) attend_tile_kernel<T, D, true, SEES><<<flat, 256, 0, s>>>(a, (int)t0, (int)n);
      else attend_tile_kernel<T, D, false, SEES><<<flat, 256, 0, s>>>(a, (int)t0, (int)n);
    }
  } else {
    dim3 g((unsigned)(rt * a.splits), (unsigned)a.c.heads, (unsigned)a.b.requests);
    if (SEES != RANGE) g = dim3((unsigned)((a.splits * a.c.heads * a.b.requests + 7) / 8 * 8 * a.row_tiles));
    constexpr int W = rows_waves(D, SEES);
    if (a.block == 16) attend_rows_kernel<T, D, 1, SEES, W><<<g, 64 * W, 0, s>>>(a);
    else if constexpr (D < 256) attend_rows_kernel<T, D, 2, SEES, W><<<g, 64 * W, 0, s>>>(a);
  }
  if (a.splits > 1) {
    const int64_t per = 256 / (D / 4), n = most_new(a) * a.c.heads * a.group;
    attend_join_kernel<T, D, SEES><<<dim3((unsigned)((n + per - 1) / per), (unsigned)a.b.requests), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <class T, int SEES>
hipError_t launch_attend_t(const AttendArgs &a, hipStream_t s) {
  switch (a.c.dim) {
    case 64: return launch_attend_d<T, 64, SEES>(a, s);
    case 96: return launch_attend_d<T, 96, SEES>(a, s);
    case 128: return launch_attend_d<T, 128, SEES>(a, s);
    default: return launch_attend_d<T, 256, SEES>(a, s);
  }
}
template <class T>
hipError_t launch_attend_s(const AttendArgs &a, hipStream_t s) {
  return a.tree.mask ? launch_attend_t<T, TREE>(a, s) : a.sinks ? launch_attend_t<T, SINKS>(a, s) : launch_attend_t<T, RANGE>(a, s);
}

}  // namespace

bool attend_plan(AttendArgs &a, int cus) {
  a.block = block_rows(a, cus);
  const int64_t rows = most_new(a) * a.group, rt = (rows + a.block - 1) / a.block;
  const int64_t base = std::max<int64_t>(1, rt * a.c.heads * a.b.requests);
  // Parts of a request's tokens, until two workgroups stand on every CU (one of 32
  // rows: its waves hold twice the accumulators; 4 requests, 5 tokens, window 8191: 24 us
  // in 8 parts, 26 in 16).  A part has two tiles or more for every wave, and what is
  // done in four is not cut at all: joining costs as much.
  const int64_t most = a.b.max_len <= 1024 ? 1 : (a.b.max_len + 511) / 512, want = (a.block == 32 ? 1 : 2) * cus;
  a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(most, 64), want / base));
  if (a.sinks || a.tree.mask) {
    const int64_t len = a.window > 0 ? std::min<int64_t>(a.b.max_len, (int64_t)a.window + (a.tree.mask ? 64 * a.tree.words : most_new(a)) + a.sinks + 128) : a.b.max_len;
    // Parts of `chunk` tiles: a request has as many as it has tokens for, so that long ones do not go on alone (16 drafts
    // of 64 behind 1000 to 16384 tokens: 222 us in up to 6 parts, 255 in 4, 292 in 2), a part two tiles or more for each wave.
    // Small blocks stand one on a CU, and joining costs more than a second gains (32 of a window of 4096: 50 us in one
    // part, 58 in two; 8 drafts of 25: 31 and 45).
    const int64_t tiles = (len + 63) / 64, least = a.block == 128 ? 32 : 2 * rows_waves(a.c.dim, SINKS);
    const int64_t parts = (a.block == 128 ? 6 : 1) * cus / base;
    a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(parts, 64), tiles / least));
    a.row_tiles = (int32_t)std::min<int64_t>(rt, 0x7fffffff);
    a.chunk = (int32_t)std::max<int64_t>(1, (tiles + a.splits - 1) / a.splits);
  }
  return (int64_t)a.splits * a.c.heads * a.b.requests <= kMaxGroups;
}

size_t attend_work_bytes(const AttendArgs &a) {
  if (a.splits == 1) return 0;
  return (size_t)a.splits * a.b.tokens * a.c.heads * a.group * (a.c.dim + 4) * sizeof(float);
}

hipError_t launch_attend(const AttendArgs &a, int type, hipStream_t s) {
  return type == PALQ_F16 ? launch_attend_s<F16>(a, s) : launch_attend_s<BF16>(a, s);
}

}  // namespace palq
