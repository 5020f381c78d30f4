// C ABI of the 8-bit transformer operators: host-side validation of every
// call, the context's workspace, and dispatch to the kernels.
#include <math.h>

#include <algorithm>
#include <new>
#include <string>

#include "cache.h"
#include "linear.h"
#include "palq_internal.h"

using namespace palq;

// Weights in slabs, their scales and bias, in one allocation.
struct palq_linear {
  palq_ctx *ctx = nullptr;
  int device = -1;
  int32_t n_out = 0, n_in = 0, kp = 0;
  int64_t max_rows = 0;
  uint8_t *mem = nullptr;
  int8_t *w = nullptr;
  float *w_scale = nullptr, *bias = nullptr;
};

namespace {

// (no exception leaves the library: without memory for the text the status stands alone)
palq_status fail(palq_ctx *ctx, palq_status code, const char *msg) {
  try {
    ctx->err = msg;
  } catch (...) {
  }
  return code;
}
palq_status device_fail(palq_ctx *ctx, hipError_t e, const char *what) {
  try {
    ctx->err = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return PALQ_ERR_DEVICE;
}

int64_t size_of(int32_t type) { return type == PALQ_F32 ? 4 : type == PALQ_I8 ? 1 : 2; }
bool floating(int32_t type) { return type == PALQ_F32 || type == PALQ_F16 || type == PALQ_BF16; }
bool aligned(const void *p, int64_t to) { return ((uintptr_t)p & (uintptr_t)(to - 1)) == 0; }
bool overlaps(const void *a, int64_t na, const void *b, int64_t nb) {
  if (!a || !b || na <= 0 || nb <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}
// Bytes from the first to the last element of `rows` rows of `cols` elements, ld apart.
int64_t extent(int64_t rows, int64_t cols, int64_t ld, int64_t size) {
  return rows <= 0 ? 0 : ((rows - 1) * ld + cols) * size;
}
// Whether a tensor's byte offsets stay far inside 63 bits.
bool sane(int64_t rows, int64_t ld) { return (double)rows * (double)ld < 1.0e17; }

constexpr int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// At least `bytes` of device memory that the next call of this kind may
// overwrite; NULL if there is none (or it would have to be allocated while the
// stream is being captured).
uint8_t *workspace(palq_ctx *ctx, size_t bytes) {
  if (bytes <= ctx->work_bytes) return ctx->work.empty() ? nullptr : ctx->work.back();
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(ctx->stream, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) return nullptr;
  const size_t twice = std::max(bytes, 2 * ctx->work_bytes);
  for (const size_t want : {twice, bytes}) {
    void *p = nullptr;
    if (hipMalloc(&p, want) == hipSuccess) {
      try {
        ctx->work.push_back((uint8_t *)p);
      } catch (...) {
        hipFree(p);
        return nullptr;
      }
      ctx->work_bytes = want;
      return (uint8_t *)p;
    }
    (void)hipGetLastError();
  }
  return nullptr;
}

// Workspace of a product: slabs of x, then its scales.
size_t linear_work(int64_t rows, int32_t kp) { return (size_t)(up(rows, kLinearRows) * ((int64_t)kp + 4)); }

palq_status check_cache(palq_ctx *ctx, const palq_cache *c) {
  if (!c) return fail(ctx, PALQ_ERR_ARG, "cache: null descriptor");
  if (c->pages < 1 || c->heads < 1) return fail(ctx, PALQ_ERR_ARG, "cache: non-positive size");
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
    return fail(ctx, PALQ_ERR_UNSUPPORTED, "cache: page_tokens not in {16,32,64,128}");
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256)
    return fail(ctx, PALQ_ERR_UNSUPPORTED, "cache: head_dim not in {64,96,128,256}");
  if (c->heads > 65535) return fail(ctx, PALQ_ERR_UNSUPPORTED, "cache: more than 65535 heads");
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(ctx, PALQ_ERR_ARG, "cache: null pointer");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(ctx, PALQ_ERR_ARG, "cache: k and v must be 16-byte aligned");
  if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
    return fail(ctx, PALQ_ERR_ARG, "cache: scales must be 4-byte aligned");
  return PALQ_OK;
}

palq_status check_batch(palq_ctx *ctx, const palq_batch *b) {
  if (!b) return fail(ctx, PALQ_ERR_ARG, "batch: null descriptor");
  if (b->requests < 0 || b->tokens < 0 || b->max_new < 0 || b->max_len < 0 || b->max_pages < 1)
    return fail(ctx, PALQ_ERR_ARG, "batch: negative size, or max_pages < 1");
  if (b->requests > 32767) return fail(ctx, PALQ_ERR_UNSUPPORTED, "batch: more than 32767 requests");
  if (b->requests > 0 && (!b->table || !b->lens || !b->starts)) return fail(ctx, PALQ_ERR_ARG, "batch: null array");
  if (!aligned(b->table, 4) || !aligned(b->lens, 4) || !aligned(b->starts, 4))
    return fail(ctx, PALQ_ERR_ARG, "batch: arrays must be 4-byte aligned");
  return PALQ_OK;
}

// A [tokens][heads][dim] tensor.
palq_status check_rows(palq_ctx *ctx, const void *p, int64_t tokens, int64_t row, int64_t head, int32_t heads, int32_t dim,
                       int32_t type) {
  if (tokens > 0 && !p) return fail(ctx, PALQ_ERR_ARG, "tensor: null pointer");
  if (!aligned(p, size_of(type))) return fail(ctx, PALQ_ERR_ARG, "tensor: not aligned to its elements");
  if (head < dim && heads > 1) return fail(ctx, PALQ_ERR_ARG, "tensor: heads overlap (stride below head_dim)");
  if (row < 0 || head < 0 || (tokens > 1 && row < dim))
    return fail(ctx, PALQ_ERR_ARG, "tensor: rows overlap (stride below head_dim)");
  if (!sane(tokens, row) || !sane(heads, head)) return fail(ctx, PALQ_ERR_ARG, "tensor: too large");
  return PALQ_OK;
}

// Whether any row (dim elements) of a tensor of rows t, heads h at t row + h head lies over another of its own, or,
// with `apart` elements between them, over one of a second tensor of the same strides.
bool rows_meet(int64_t tokens, int64_t row, int32_t heads, int64_t head, int32_t dim, int64_t apart, bool own) {
  const int64_t cols = (heads - 1) * head + dim, all = (tokens - 1) * row + cols, gap = apart < 0 ? -apart : apart;
  if (own ? row >= cols || head >= (tokens - 1) * row + dim : gap >= all || (gap >= cols && row >= gap + cols)) return false;
  for (int64_t h = own ? 0 : 1 - heads; h < heads; ++h) {
    // t row + h head + apart within (-dim, dim) for a t of (-tokens, tokens)
    const int64_t off = h * head + apart;
    if (tokens == 1 || row == 0) {
      if (off > -dim && off < dim && !(own && h == 0)) return true;
      continue;
    }
    for (int64_t t = -off / row - 1; t <= -off / row + 1; ++t)
      if (t > -tokens && t < tokens && !(own && h == 0 && t == 0) && t * row + off > -dim && t * row + off < dim) return true;
  }
  return false;
}

// Tensors that a call writes: no two rows over each other, none over the cache.
palq_status check_written(palq_ctx *ctx, const palq_cache *c, const void *p, int64_t tokens, int64_t row, int64_t head,
                          int32_t heads, int32_t type) {
  if (tokens <= 0) return PALQ_OK;
  if (rows_meet(tokens, row, heads, head, c->head_dim, 0, true)) return fail(ctx, PALQ_ERR_ARG, "output: rows overlap");
  const int64_t bytes = ((tokens - 1) * row + (heads - 1) * head + c->head_dim) * size_of(type);
  const int64_t blocks = (int64_t)c->pages * c->heads, codes = blocks * c->page_tokens * c->head_dim;
  if (overlaps(p, bytes, c->k, codes) || overlaps(p, bytes, c->v, codes) || overlaps(p, bytes, c->k_scale, blocks * 4) ||
      overlaps(p, bytes, c->v_scale, blocks * 4))
    return fail(ctx, PALQ_ERR_ARG, "output: overlaps the cache");
  return PALQ_OK;
}

CacheView view_of(const palq_cache *c) {
  CacheView v{c->k, c->v, c->k_scale, c->v_scale, c->pages, c->heads, c->head_dim, c->page_tokens, 0};
  while ((1 << v.shift) < v.page) ++v.shift;
  return v;
}
BatchView view_of(const palq_cache *c, const palq_batch *b) {
  const int64_t limit = std::min(std::min((int64_t)b->max_pages * c->page_tokens, (int64_t)b->max_len), kMaxTokens);
  return BatchView{b->table, b->lens, b->starts, b->requests, b->max_pages, b->max_new, b->tokens, b->max_len,
                   (int32_t)std::min(b->tokens, (int64_t)0x7fffffff), (int32_t)limit};
}

}  // namespace

extern "C" {

palq_status palq_quantize_rows(palq_ctx *ctx, const void *x, int32_t type, int64_t rows, int32_t cols, int64_t x_ld,
                               int8_t *codes, int64_t codes_ld, float *scales) {
  if (!ctx) return PALQ_ERR_ARG;
  if (!floating(type)) return fail(ctx, PALQ_ERR_ARG, "quantize rows: type must be PALQ_F32, F16 or BF16");
  if (rows < 0 || cols < 1 || x_ld < cols || codes_ld < cols) return fail(ctx, PALQ_ERR_ARG, "quantize rows: sizes");
  if (rows >= (int64_t)1 << 31) return fail(ctx, PALQ_ERR_UNSUPPORTED, "quantize rows: 2^31 rows or more");
  if (cols > 0x7ffffff0) return fail(ctx, PALQ_ERR_UNSUPPORTED, "quantize rows: row too long");
  if (!sane(rows, x_ld) || !sane(rows, codes_ld)) return fail(ctx, PALQ_ERR_ARG, "quantize rows: tensor too large");
  if (rows > 0 && (!x || !codes || !scales)) return fail(ctx, PALQ_ERR_ARG, "quantize rows: null pointer");
  if (!aligned(x, size_of(type)) || !aligned(scales, 4)) return fail(ctx, PALQ_ERR_ARG, "quantize rows: misaligned pointer");
  const int64_t xb = extent(rows, cols, x_ld, size_of(type)), cb = extent(rows, cols, codes_ld, 1);
  if (overlaps(x, xb, codes, cb) || overlaps(x, xb, scales, rows * 4) || overlaps(codes, cb, scales, rows * 4))
    return fail(ctx, PALQ_ERR_ARG, "quantize rows: x, codes and scales overlap");
  if (ctx->device < 0 || rows == 0) return PALQ_OK;
  hipSetDevice(ctx->device);
  const hipError_t e = launch_quantize_rows(x, type, rows, cols, x_ld, (cols + 15) / 16 * 16, codes, codes_ld, false, scales,
                                            ctx->stream);
  return e == hipSuccess ? PALQ_OK : device_fail(ctx, e, "quantize rows");
}

palq_status palq_linear_create(palq_ctx *ctx, const int8_t *w, int64_t w_ld, const float *w_scale, const float *bias,
                               int32_t n_out, int32_t n_in, int64_t max_rows, palq_linear **out) {
  if (!ctx) return PALQ_ERR_ARG;
  if (!out) return fail(ctx, PALQ_ERR_ARG, "linear: null out");
  *out = nullptr;
  if (n_out < 1 || n_in < 1 || w_ld < n_in || max_rows < 0) return fail(ctx, PALQ_ERR_ARG, "linear: sizes");
  if (!w || !w_scale) return fail(ctx, PALQ_ERR_ARG, "linear: null weights or scales");
  if (!aligned(w_scale, 4) || !aligned(bias, 4)) return fail(ctx, PALQ_ERR_ARG, "linear: scales and bias must be 4-byte aligned");
  if (n_in >= 1 << 17) return fail(ctx, PALQ_ERR_OVERFLOW, "linear: n_in >= 2^17, the int32 sum could overflow");
  if (n_out > 1 << 24 || max_rows > 1 << 24) return fail(ctx, PALQ_ERR_UNSUPPORTED, "linear: more than 2^24 channels or rows");
  if (!sane(n_out, w_ld)) return fail(ctx, PALQ_ERR_ARG, "linear: weights too large");
  palq_linear *l = new (std::nothrow) palq_linear();
  if (!l) return fail(ctx, PALQ_ERR_NOMEM, "linear: host memory");
  l->ctx = ctx;
  l->device = ctx->device;
  l->n_out = n_out;
  l->n_in = n_in;
  l->kp = (int32_t)up(n_in, kLinearK);
  l->max_rows = max_rows;
  if (ctx->device < 0) {
    *out = l;
    return PALQ_OK;
  }
  hipSetDevice(ctx->device);
  const int64_t np = up(n_out, kLinearRows), wb = np * l->kp;
  if (hipMalloc((void **)&l->mem, (size_t)(wb + 8 * np)) != hipSuccess) {
    (void)hipGetLastError();
    delete l;
    return fail(ctx, PALQ_ERR_NOMEM, "linear: weights");
  }
  l->w = (int8_t *)l->mem;
  l->w_scale = (float *)(l->mem + wb);
  if (bias) l->bias = l->w_scale + np;
  hipError_t e = launch_slabs(w, n_out, np, n_in, w_ld, l->kp, l->w, ctx->stream);
  if (e == hipSuccess) e = hipMemcpyAsync(l->w_scale, w_scale, (size_t)n_out * 4, hipMemcpyDeviceToDevice, ctx->stream);
  if (e == hipSuccess && bias) e = hipMemcpyAsync(l->bias, bias, (size_t)n_out * 4, hipMemcpyDeviceToDevice, ctx->stream);
  if (e == hipSuccess) e = hipStreamSynchronize(ctx->stream);
  if (e != hipSuccess) {
    palq_linear_destroy(l);
    return device_fail(ctx, e, "linear: weights");
  }
  if (max_rows > 0 && !workspace(ctx, linear_work(max_rows, l->kp))) {
    palq_linear_destroy(l);
    return fail(ctx, PALQ_ERR_NOMEM, "linear: workspace");
  }
  *out = l;
  return PALQ_OK;
}

palq_status palq_linear_run(palq_ctx *ctx, const palq_linear *lin, const void *x, int32_t x_type, int64_t x_ld,
                            const float *x_scale, int64_t rows, void *y, int32_t y_type, int64_t y_ld) {
  if (!ctx) return PALQ_ERR_ARG;
  if (!lin) return fail(ctx, PALQ_ERR_ARG, "linear: null layer");
  if (lin->ctx != ctx) return fail(ctx, PALQ_ERR_ARG, "linear: layer of another context");
  if (!floating(x_type) && x_type != PALQ_I8) return fail(ctx, PALQ_ERR_ARG, "linear: unknown x type");
  if (!floating(y_type)) return fail(ctx, PALQ_ERR_ARG, "linear: y type must be PALQ_F32, F16 or BF16");
  if (rows < 0 || rows > lin->max_rows) return fail(ctx, PALQ_ERR_ARG, "linear: rows outside [0, max_rows]");
  if (x_ld < lin->n_in || y_ld < lin->n_out) return fail(ctx, PALQ_ERR_ARG, "linear: row stride below the row");
  if (rows > 0 && (!x || !y)) return fail(ctx, PALQ_ERR_ARG, "linear: null pointer");
  if (rows > 0 && (x_type == PALQ_I8) != (x_scale != nullptr))
    return fail(ctx, PALQ_ERR_ARG, "linear: x_scale goes with codes (PALQ_I8) and with nothing else");
  if (!aligned(x, size_of(x_type)) || !aligned(y, size_of(y_type)) || !aligned(x_scale, 4))
    return fail(ctx, PALQ_ERR_ARG, "linear: pointer not aligned to its elements");
  if (!sane(rows, x_ld) || !sane(rows, y_ld)) return fail(ctx, PALQ_ERR_ARG, "linear: tensor too large");
  const int64_t yb = extent(rows, lin->n_out, y_ld, size_of(y_type));
  if (overlaps(x, extent(rows, lin->n_in, x_ld, size_of(x_type)), y, yb) || overlaps(x_scale, rows * 4, y, yb))
    return fail(ctx, PALQ_ERR_ARG, "linear: y overlaps an input");
  if (ctx->device < 0 || rows == 0) return PALQ_OK;
  hipSetDevice(ctx->device);
  uint8_t *work = workspace(ctx, linear_work(rows, lin->kp));
  if (!work) return fail(ctx, PALQ_ERR_NOMEM, "linear: workspace");
  const int64_t padded = up(rows, kLinearRows);
  LinearArgs a{(int8_t *)work, lin->w, (float *)(work + padded * lin->kp), lin->w_scale, lin->bias, y, rows, y_ld,
               lin->n_out, lin->kp};
  hipError_t e;
  if (x_type != PALQ_I8 && linear_one(rows, lin->kp)) {
    e = launch_linear_one(a, x, x_type, lin->n_in, y_type, ctx->stream);
    return e == hipSuccess ? PALQ_OK : device_fail(ctx, e, "linear");
  }
  if (x_type == PALQ_I8) {
    e = launch_slabs((const int8_t *)x, rows, up(rows, 16), lin->n_in, x_ld, lin->kp, (int8_t *)work, ctx->stream);
    a.x_scale = x_scale;
  } else {
    e = launch_quantize_rows(x, x_type, rows, lin->n_in, x_ld, lin->kp, (int8_t *)work, 0, true, (float *)a.x_scale,
                             ctx->stream);
  }
  if (e == hipSuccess) e = launch_linear(a, y_type, ctx->stream);
  return e == hipSuccess ? PALQ_OK : device_fail(ctx, e, "linear");
}

void palq_linear_destroy(palq_linear *lin) {
  if (!lin) return;
  if (lin->mem) {
    hipSetDevice(lin->device);
    hipFree(lin->mem);
  }
  delete lin;
}

const char *palq_linear_kernels(const palq_linear *lin, int64_t rows) {
  if (!lin) return nullptr;
  return lin->device < 0 ? "" : linear_kernel_label(rows, lin->n_out, lin->kp);
}

palq_status palq_cache_append(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, const void *k, int64_t k_row,
                              int64_t k_head, const void *v, int64_t v_row, int64_t v_head, int32_t type) {
  if (!ctx) return PALQ_ERR_ARG;
  palq_status st;
  if ((st = check_cache(ctx, cache)) || (st = check_batch(ctx, batch))) return st;
  if (!floating(type)) return fail(ctx, PALQ_ERR_ARG, "append: type must be PALQ_F32, F16 or BF16");
  if ((st = check_rows(ctx, k, batch->tokens, k_row, k_head, cache->heads, cache->head_dim, type)) ||
      (st = check_rows(ctx, v, batch->tokens, v_row, v_head, cache->heads, cache->head_dim, type)))
    return st;
  if (ctx->device < 0 || batch->requests == 0 || batch->tokens == 0 || batch->max_new == 0 || batch->max_len == 0)
    return PALQ_OK;
  hipSetDevice(ctx->device);
  const int64_t stride[4] = {k_row, k_head, v_row, v_head};
  const hipError_t e = launch_cache_append(view_of(cache), view_of(cache, batch), k, v, type, stride, ctx->stream);
  return e == hipSuccess ? PALQ_OK : device_fail(ctx, e, "cache append");
}

palq_status palq_cache_read(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, void *k, int64_t k_row,
                            int64_t k_head, void *v, int64_t v_row, int64_t v_head, int32_t type) {
  if (!ctx) return PALQ_ERR_ARG;
  palq_status st;
  if ((st = check_cache(ctx, cache)) || (st = check_batch(ctx, batch))) return st;
  if (!floating(type)) return fail(ctx, PALQ_ERR_ARG, "cache read: type must be PALQ_F32, F16 or BF16");
  if ((st = check_rows(ctx, k, batch->tokens, k_row, k_head, cache->heads, cache->head_dim, type)) ||
      (st = check_rows(ctx, v, batch->tokens, v_row, v_head, cache->heads, cache->head_dim, type)))
    return st;
  if ((st = check_written(ctx, cache, k, batch->tokens, k_row, k_head, cache->heads, type)) ||
      (st = check_written(ctx, cache, v, batch->tokens, v_row, v_head, cache->heads, type)))
    return st;
  if (batch->tokens > 0) {  // (k and v may share rows of a fused tensor, but no element)
    const int64_t apart = (const char *)v - (const char *)k, size = size_of(type);
    const bool alike = k_row == v_row && k_head == v_head;
    if (alike ? rows_meet(batch->tokens, k_row, cache->heads, k_head, cache->head_dim, apart / size, false)
              : apart > -cache->head_dim * size && apart < cache->head_dim * size)
      return fail(ctx, PALQ_ERR_ARG, "cache read: k and v overlap");
  }
  if (ctx->device < 0 || batch->requests == 0 || batch->tokens == 0 || batch->max_new == 0 || batch->max_len == 0)
    return PALQ_OK;
  hipSetDevice(ctx->device);
  const int64_t stride[4] = {k_row, k_head, v_row, v_head};
  const hipError_t e = launch_cache_read(view_of(cache), view_of(cache, batch), k, v, type, stride, ctx->stream);
  return e == hipSuccess ? PALQ_OK : device_fail(ctx, e, "cache read");
}

palq_status palq_attention(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, const void *q, int64_t q_row,
                           int64_t q_head, int32_t q_heads, void *out, int64_t out_row, int64_t out_head, int32_t type,
                           float scale, int32_t causal, int32_t window) {
  if (!ctx) return PALQ_ERR_ARG;
  palq_status st;
  if ((st = check_cache(ctx, cache)) || (st = check_batch(ctx, batch))) return st;
  if (type != PALQ_F16 && type != PALQ_BF16) return fail(ctx, PALQ_ERR_ARG, "attention: type must be PALQ_F16 or PALQ_BF16");
  if (q_heads < 1 || q_heads % cache->heads) return fail(ctx, PALQ_ERR_ARG, "attention: q_heads is no multiple of the cache's heads");
  if ((st = check_rows(ctx, q, batch->tokens, q_row, q_head, q_heads, cache->head_dim, type)) ||
      (st = check_rows(ctx, out, batch->tokens, out_row, out_head, q_heads, cache->head_dim, type)))
    return st;
  if (!isfinite(scale)) return fail(ctx, PALQ_ERR_ARG, "attention: scale must be finite");
  if ((causal != 0 && causal != 1) || window < 0) return fail(ctx, PALQ_ERR_ARG, "attention: causal must be 0 or 1, window >= 0");
  if (window > 0 && !causal) return fail(ctx, PALQ_ERR_ARG, "attention: a window needs causal = 1");
  const int32_t group = q_heads / cache->heads;
  if ((int64_t)batch->max_new * group >= (int64_t)1 << 30)
    return fail(ctx, PALQ_ERR_UNSUPPORTED, "attention: 2^30 or more rows of a cache head");
  auto bytes = [&](int64_t row, int64_t head) {
    return batch->tokens <= 0 ? 0 : ((batch->tokens - 1) * row + (q_heads - 1) * head + cache->head_dim) * size_of(type);
  };
  if (overlaps(q, bytes(q_row, q_head), out, bytes(out_row, out_head)))
    return fail(ctx, PALQ_ERR_ARG, "attention: out overlaps q");
  if ((st = check_written(ctx, cache, out, batch->tokens, out_row, out_head, q_heads, type))) return st;
  if (ctx->device < 0 || batch->requests == 0 || batch->tokens == 0 || batch->max_new == 0) return PALQ_OK;
  hipSetDevice(ctx->device);
  AttendArgs a{view_of(cache), view_of(cache, batch), (const uint16_t *)q, (uint16_t *)out, q_row, q_head, out_row, out_head,
               group, causal, window, scale, 0, 1, nullptr};
  if (a.b.max_new > batch->tokens) a.b.max_new = (int32_t)batch->tokens;
  if (!attend_plan(a, ctx->cus)) return fail(ctx, PALQ_ERR_UNSUPPORTED, "attention: 2^24 or more pairs of a request and a cache head");
  if (const size_t need = attend_work_bytes(a)) {
    a.part = (float *)workspace(ctx, need);
    if (!a.part) return fail(ctx, PALQ_ERR_NOMEM, "attention: workspace (in a capture: run the shape once before)");
  }
  const hipError_t e = launch_attend(a, type, ctx->stream);
  return e == hipSuccess ? PALQ_OK : device_fail(ctx, e, "attention");
}

}  // extern "C"
