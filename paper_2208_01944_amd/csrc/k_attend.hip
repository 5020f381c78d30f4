// Attention over the paged 8-bit cache:
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j,  k_j = code ks[block], v_j = code vs[block]
// over the tokens j that query i sees (its own position and earlier ones, or a
// window of them, or all).
//
// Scores and sums are fp32.  The codes are exact in fp16, so q is the only
// operand that is rounded: each row is scaled by a power of two that brings its
// largest element to [1, 2) (bf16 values, 8 bits, stay exact but for elements
// 2^-15 below the row's largest), and the scale of a block multiplies the
// finished dot product.  Probabilities are rounded to fp16 (11 bits) as the
// second product's operand.
//
// Value scales ride in the exponent: with u_j = log2(vs), w_j = exp2(s_j + u_j -
// M), M the running maximum of s_j + u_j, the output is sum w_j code_j / L, L =
// sum w_j / vs, so every weight is at most 1 whatever the blocks' scales are,
// and no product with vs is left.  (Scales are at least 2^-100, so 1 / vs and L
// stay finite.)
//
// Matrix layout.  S^T = K Q^T with v_mfma_f32_16x16x32_f16: a lane ends up with
// scores of one query (lane % 16) and, row 4 c + i of subtile j standing for
// token 16 c + 4 j + i (c = lane / 16), with 16 consecutive tokens: all of one
// page, with one pair of scales, and in the order in which O^T = V^T P^T takes
// them as its second operand.  So probabilities never leave their lane, and V,
// stored channel by channel, is read 16 tokens at a time.
#include <algorithm>

#include "cache.h"

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
__device__ __forceinline__ h8 codes_h8(uint32_t x, uint32_t y) {
  h2 a, b, c, d;
  codes_h4(x, a, b);
  codes_h4(y, c, d);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// One row's reach: tokens [lo, hi).
struct Reach { int lo, hi; };
__device__ __forceinline__ Reach reach_of(const AttendArgs &a, const Request &q, int t) {
  const int pos = q.len - q.n + t;
  Reach s{0, q.len};
  if (a.causal) {
    s.hi = max(0, min(q.len, pos + 1));
    if (a.window > 0) s.lo = max(0, pos - a.window + 1);
  }
  return s;
}

__device__ __forceinline__ float load_half(const uint16_t *p, bool bf16) { return bf16 ? BF16::get(*p) : F16::get(*p); }

// A wave's queries: 16 columns, this lane's channels cc D / 4 .. of column
// lane % 16, scaled to fp16; returns the scale taken out.
template <class T, int D>
__device__ __forceinline__ float load_q(const uint16_t *p, bool live, bool vec, h8 *out) {
  float v[D / 4];
  uint32_t mag = 0;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    if (live && vec) {
      const v4i x = ((const v4i *)p)[s];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[8 * s + 2 * i] = T::get((uint16_t)((uint32_t)x[i] & 0xffffu));
        v[8 * s + 2 * i + 1] = T::get((uint16_t)((uint32_t)x[i] >> 16));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[8 * s + i] = live ? T::get(p[8 * s + i]) : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < D / 4; ++i) mag = max(mag, mag_bits(v[i]));
  mag = max(mag, (uint32_t)__shfl_xor((int)mag, 16));
  mag = max(mag, (uint32_t)__shfl_xor((int)mag, 32));
  const int e = max(1, (int)(mag >> 23));  // 2^(e - 127) <= largest; 255: not finite
  // a row with inf or NaN: inf 0 = NaN, so all its scores are NaN
  const float f = e == 255 ? 0.0f : __uint_as_float((uint32_t)(254 - min(e, 253)) << 23);
#pragma unroll
  for (int s = 0; s < D / 32; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) out[s][i] = (_Float16)(v[8 * s + i] * f);
  return __uint_as_float((uint32_t)min(e, 253) << 23);
}

// NQ tiles of 16 (query, head) rows a wave, 4 waves a workgroup, each wave every
// fourth tile of 64 tokens; the waves join in LDS.  Splits join in attend_join_kernel.
template <class T, int D, int NQ>
__global__ __launch_bounds__(256) void attend_rows_kernel(AttendArgs a) {
  constexpr int KS = D / 32, DT = D / 16, OLD = D + 4;
  __shared__ float sm[4][NQ * 16], sl[4][NQ * 16];
  __shared__ __attribute__((aligned(16))) float so[4][16 * OLD];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, c = lane >> 4;
  const int h = blockIdx.y, r = blockIdx.z, split = blockIdx.x % a.splits, rt = blockIdx.x / a.splits;
  const CacheView &cv = a.c;
  const Request q = request_of(a.b, r, cv.shift);
  const int rows = q.n * a.group, first = rt * NQ * 16;
  if (first >= rows) return;
  const int last = min(rows, first + NQ * 16) - 1;

  // tokens that any of the tile's rows sees, in tiles of 64
  const Reach rf = reach_of(a, q, first / a.group), rl = reach_of(a, q, last / a.group);
  const int lo = rf.lo, hi = rl.hi;
  const int tile0 = lo >> 6, ntiles = hi > lo ? ((hi + 63) >> 6) - tile0 : 0;
  const int per = (ntiles + a.splits - 1) / a.splits;
  const int tb = tile0 + min(ntiles, split * per), te = tile0 + min(ntiles, (split + 1) * per);

  h8 Q[NQ][KS];
  float f[NQ];
  int rlo[NQ], rhi[NQ];
  const bool vec = (((uintptr_t)a.q | (uintptr_t)(a.q_row * 2) | (uintptr_t)(a.q_head * 2)) & 15u) == 0;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int row = first + n * 16 + col;
    const bool live = row < rows;
    const int t = live ? row / a.group : 0, g = live ? row - t * a.group : 0;
    const uint16_t *p = a.q + (q.row0 + t) * a.q_row + (int64_t)(h * a.group + g) * a.q_head + c * (D / 4);
    f[n] = load_q<T, D>(p, live, vec, Q[n]) * a.scale;
    const Reach s = reach_of(a, q, t);
    rlo[n] = s.lo;
    rhi[n] = live ? s.hi : 0;
  }
  v4f O[NQ][DT];
  float M[NQ], L[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    M[n] = -INFINITY;
    L[n] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) O[n][d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int32_t *table = a.b.table + (int64_t)r * a.b.max_pages;
  // page of the 16 tokens from `tok` on; -1: no such page
  auto page_at = [&](int tok) __attribute__((always_inline)) {
    if (tok >= hi) return -1;
    const int pid = table[tok >> cv.shift];
    return pid >= 0 && pid < cv.pages ? pid : -1;
  };
  const int pm = cv.page - 1;
  for (int tile = tb + wave; tile < te; tile += 4) {
    const int t0 = tile << 6;
    const int kt = t0 + (col >> 2) * 16, vt = t0 + c * 16;  // first token of the chunks this lane loads
    const int kp = page_at(kt), vp = page_at(vt);
    const int8_t *kb = cv.k + (((int64_t)max(kp, 0) * cv.heads + h) * cv.page + (kt & pm) + (col & 3)) * D + c * (D / 4);
    const int8_t *vb = cv.v + (((int64_t)max(vp, 0) * cv.heads + h) * D + col) * cv.page + (vt & pm);
    const int64_t sc = (int64_t)max(vp, 0) * cv.heads + h;
    const float ks = cv.ks[sc], vs = cv.vs[sc];
    uint32_t kx[4][D / 16];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int w = 0; w < D / 32; ++w) {
        const v2i x = *(const v2i *)(kb + (int64_t)j * 4 * D + w * 8);
        kx[j][2 * w] = (uint32_t)x[0];
        kx[j][2 * w + 1] = (uint32_t)x[1];
      }
    v4i vx[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) vx[d] = *(const v4i *)(vb + (int64_t)d * 16 * cv.page);
    v4f S[NQ][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) S[n][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const h8 A = codes_h8(kx[j][2 * s], kx[j][2 * s + 1]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) S[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, Q[n][s], S[n][j], 0, 0, 0);
      }
    }
    const float u = __builtin_log2f(vs), rv = 1.0f / vs;
    h8 P[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float fk = f[n] * ks;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = vt + 4 * j + i;
          const bool sees = tok >= rlo[n] && tok < rhi[n] && vp >= 0;
          const float s = sees ? __builtin_fmaf(S[n][j][i], fk, u) : -INFINITY;
          S[n][j][i] = s;
          mx = fmaxf(mx, s);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(M[n], mx), ms = mn == -INFINITY ? 0.0f : mn;
      const float alpha = exp2_fast(M[n] - ms);
      M[n] = mn;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(S[n][j][i] - ms);
          sum += p;
          P[n][j >> 1][(j & 1) * 4 + i] = (_Float16)p;
        }
      L[n] = L[n] * alpha + (sum == 0.0f ? 0.0f : sum * rv);
      if (!__all(alpha == 1.0f))
#pragma unroll
        for (int d = 0; d < DT; ++d) O[n][d] *= alpha;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const h8 A = codes_h8((uint32_t)vx[d][2 * s], (uint32_t)vx[d][2 * s + 1]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) O[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, P[n][s], O[n][d], 0, 0, 0);
      }
  }

  // the waves' results under one maximum
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
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int rc = n * 16 + col;
    const float mt = fmaxf(fmaxf(sm[0][rc], sm[1][rc]), fmaxf(sm[2][rc], sm[3][rc]));
    const float wgt = exp2_fast(M[n] - (mt == -INFINITY ? 0.0f : mt));
#pragma unroll
    for (int d = 0; d < DT; ++d) *(v4f *)&so[wave][col * OLD + d * 16 + c * 4] = O[n][d] * wgt;
    __syncthreads();
    for (int p = threadIdx.x; p < 16 * (D / 4); p += 256) {
      const int qr = p / (D / 4), d = p % (D / 4) * 4, row = first + n * 16 + qr;
      if (row >= rows) continue;
      const int t = row / a.group, hq = h * a.group + row - t * a.group;
      v4f o = *(v4f *)&so[0][qr * OLD + d];
#pragma unroll
      for (int w = 1; w < 4; ++w) o += *(v4f *)&so[w][qr * OLD + d];
      const int rq = n * 16 + qr;
      float m = -INFINITY, l = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) m = fmaxf(m, sm[w][rq]);
#pragma unroll
      for (int w = 0; w < 4; ++w) l += sl[w][rq] * exp2_fast(sm[w][rq] - (m == -INFINITY ? 0.0f : m));
      if (a.splits == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const float v[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        uint16_t *dst = a.out + (q.row0 + t) * a.out_row + (int64_t)hq * a.out_head + d;
        store4<T>(dst, v, (((uintptr_t)a.out | (uintptr_t)(a.out_row * 2) | (uintptr_t)(a.out_head * 2)) & 7u) == 0);
      } else {
        const int64_t hs = (int64_t)cv.heads * a.group;
        const int64_t at = ((int64_t)split * a.b.tokens + q.row0 + t) * hs + hq;
        *(v4f *)(a.part + at * D + d) = o;
        if (d == 0) {
          float *ml = a.part + (int64_t)a.splits * a.b.tokens * hs * D + at * 2;
          ml[0] = m;
          ml[1] = l;
        }
      }
    }
    __syncthreads();
  }
}

// One (token, head) row a group of D / 4 threads: the splits under one maximum.
template <class T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int W = D / 4;
  const int r = blockIdx.y;
  const Request q = request_of(a.b, r, a.c.shift);
  const int hs = a.c.heads * a.group, sub = threadIdx.x / W, d = threadIdx.x % W * 4;
  const int64_t i = (int64_t)blockIdx.x * (256 / W) + sub;
  if (sub >= 256 / W || i >= (int64_t)q.n * hs) return;
  const int64_t t = i / hs, hq = i - t * hs, at = (q.row0 + t) * hs + hq, step = a.b.tokens * hs;
  const float *ml = a.part + a.splits * step * D;
  float m = -INFINITY, l = 0.0f;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, ml[(s * step + at) * 2]);
  const float ms = m == -INFINITY ? 0.0f : m;
  v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < a.splits; ++s) {
    const float w = exp2_fast(ml[(s * step + at) * 2] - ms);
    l += ml[(s * step + at) * 2 + 1] * w;
    o += *(const v4f *)(a.part + (s * step + at) * D + d) * w;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const float v[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  uint16_t *dst = a.out + (q.row0 + t) * a.out_row + hq * a.out_head + d;
  store4<T>(dst, v, (((uintptr_t)a.out | (uintptr_t)(a.out_row * 2) | (uintptr_t)(a.out_head * 2)) & 7u) == 0);
}

// Row tiles of a workgroup in the kernel's NQ.
int row_tiles(const AttendArgs &a) {
  const int64_t rows = (int64_t)a.b.max_new * a.group;
  return rows <= 16 ? 1 : rows <= 32 || a.c.dim == 256 ? 2 : 4;
}

template <class T, int D>
hipError_t launch_attend_d(const AttendArgs &a, hipStream_t s) {
  const int nq = row_tiles(a);
  const int64_t rows = (int64_t)a.b.max_new * a.group;
  const dim3 g((unsigned)((rows + nq * 16 - 1) / (nq * 16) * a.splits), (unsigned)a.c.heads, (unsigned)a.b.requests);
  if (nq == 1) attend_rows_kernel<T, D, 1><<<g, 256, 0, s>>>(a);
  else if (nq == 2) attend_rows_kernel<T, D, 2><<<g, 256, 0, s>>>(a);
  else if constexpr (D < 256) attend_rows_kernel<T, D, 4><<<g, 256, 0, s>>>(a);
  if (a.splits > 1) {
    const int64_t per = 256 / (D / 4), n = (int64_t)a.b.max_new * a.c.heads * a.group;
    attend_join_kernel<T, D><<<dim3((unsigned)((n + per - 1) / per), (unsigned)a.b.requests), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <class T>
hipError_t launch_attend_t(const AttendArgs &a, hipStream_t s) {
  switch (a.c.dim) {
    case 64: return launch_attend_d<T, 64>(a, s);
    case 96: return launch_attend_d<T, 96>(a, s);
    case 128: return launch_attend_d<T, 128>(a, s);
    default: return launch_attend_d<T, 256>(a, s);
  }
}

}  // namespace

void attend_plan(AttendArgs &a, int cus) {
  const int64_t rows = (int64_t)a.b.max_new * a.group, nq = row_tiles(a) * 16;
  const int64_t base = std::max<int64_t>(1, (rows + nq - 1) / nq * a.c.heads * a.b.requests);
  // every wave at least one tile of 64 tokens
  const int64_t most = std::max<int64_t>(1, (a.b.max_len + 255) / 256);
  a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(most, 64), 2 * cus / base));
}

size_t attend_work_bytes(const AttendArgs &a) {
  if (a.splits == 1) return 0;
  return (size_t)a.splits * a.b.tokens * a.c.heads * a.group * (a.c.dim + 2) * sizeof(float);
}

hipError_t launch_attend(const AttendArgs &a, int type, hipStream_t s) {
  return type == PALQ_F16 ? launch_attend_t<F16>(a, s) : launch_attend_t<BF16>(a, s);
}

}  // namespace palq
