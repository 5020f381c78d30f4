/*
 * palq.h -- C ABI of the PalQuant inference library for AMD MI355X (gfx950).
 *
 * PalQuant (parallel low-precision quantisation) runs a high-precision
 * network as G parallel groups of B-bit convolutions (Section 4.1), with a
 * cyclic permutation of the groups between layers (Section 4.2, Eq. 6-8).
 * This library computes the integer inference path of such a network on one
 * GPU: quantise (Eq. 2), grouped B-bit convolution with int32 accumulation
 * (Eq. 1 per group), a fixed-point requantisation with ReLU, and the cyclic
 * permutation applied as the write address of the result.
 *
 * Conventions for every call
 *  - Tensor and parameter pointers are DEVICE pointers owned by the caller
 *    unless a comment says "host".  The library never frees them.
 *  - Calls are asynchronous on the context's stream.  All argument checks
 *    happen on the host before anything is enqueued: a call that returns an
 *    error other than PALQ_ERR_DEVICE has written nothing.  Device faults
 *    surface on a later call or on palq_sync.
 *  - No call throws or aborts across the ABI.  palq_last_error() gives a
 *    human-readable reason for the last failing call on that context.
 *  - A context is used by one host thread at a time.
 *  - A context created with device = -1 is "validate only": every call checks
 *    its arguments exactly as on a GPU and then returns without device work.
 *
 * Packed code layout (activations and filters)
 *  A tensor [N][H][W][G][C^] of b-bit codes is stored NHWC, group-major
 *  (channel g*C^ + j, the [N, G, C^, H, W] view of Section 4.2).  Each
 *  (pixel, group) row of C^ codes occupies palq_row_bytes(C^, b) bytes and
 *  rows follow each other with no gap; a pixel is G rows.  That is layout
 *  PALQ_LAYOUT_PIXEL.  PALQ_LAYOUT_GROUP stores the same rows as
 *  [G][N][H][W]: all of group 0's rows in pixel order, then group 1's, ...
 *  (a group's rows of consecutive pixels are adjacent, so one group's tile
 *  of pixels is one contiguous run).  Both take palq_act_bytes() bytes.
 *   - b in {2, 4, 8}: code j sits at bits [b*j, b*j + b) of the row read as
 *     one little-endian bit string; the row is padded with zero bits to a
 *     multiple of 32 bits.
 *   - b = 6: stored as b = 8 (code j in bits 0-5 of byte j, bits 6-7 zero),
 *     for dense 6-bit baselines.
 *   - b = 3: the row is cut into chunks of 32 codes (the last one padded with
 *     zero codes), 12 bytes each.  In a chunk, bytes 0-7 are a little-endian
 *     64-bit field holding bits 0-1 of code j at bits [2j, 2j+2); bytes 8-11
 *     are a little-endian 32-bit field holding bit 2 of code j at bit
 *     2*(j & 15) + (j >> 4) (codes 0-15 at the even bits, 16-31 at the odd
 *     bits).
 *  Signed codes are b-bit two's complement, unsigned codes are plain binary.
 *  Padding bits are written as zero and ignored when read.
 *  A filter [G][C^out][kh][kw][C^in] has the layout of an activation tensor
 *  with N = G*C^out, H = kh, W = kw and one group of C^in codes.
 */
#ifndef PALQ_H
#define PALQ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t palq_status;
#define PALQ_OK 0
#define PALQ_ERR_ARG (-1)         /* malformed or inconsistent arguments        */
#define PALQ_ERR_UNSUPPORTED (-2) /* well formed but outside what is built      */
#define PALQ_ERR_OVERFLOW (-3)    /* the int32 accumulator bound could be broken */
#define PALQ_ERR_DEVICE (-4)      /* HIP runtime error                          */
#define PALQ_ERR_NOMEM (-5)       /* device or host allocation failed           */

typedef struct palq_ctx palq_ctx;
typedef struct palq_net palq_net;

/* An activation tensor: n x h x w pixels of `groups` rows of ch_per_group
 * codes, `bits` in {2, 3, 4, 6, 8}.  data: device, palq_act_bytes() bytes.
 * layout: PALQ_LAYOUT_PIXEL (0, what a zeroed descriptor holds) or
 * PALQ_LAYOUT_GROUP (see the packed code layout above); every call takes
 * either, and the tensors of one call may mix them. */
#define PALQ_LAYOUT_PIXEL 0
#define PALQ_LAYOUT_GROUP 1
typedef struct {
  int32_t n, h, w;
  int32_t groups, ch_per_group;
  int32_t bits;
  int32_t is_signed;
  int32_t layout;
  void *data;
} palq_act;

/* A grouped filter: groups x cout_pg output channels, each a kh x kw x
 * cin_pg block of signed `bits`-bit codes (bits in {2, 3, 4, 6, 8}).
 * data: device, packed as described above. */
typedef struct {
  int32_t groups, cout_pg, cin_pg, kh, kw, bits;
  const void *data;
} palq_filter;

/* Per-output-channel fixed-point requantisation, arrays of groups*cout_pg
 * int32 on the device, indexed by the convolution's own output channel
 * g*cout_pg + k (before the cyclic permutation moves it):
 *   q = clamp(floor((t * mult + 2^(shift-1)) / 2^shift), 0, 2^out_bits - 1)
 * with t = acc + bias + residual (below).  The clamp at 0 is the fused ReLU.
 * The result is exact for mult in [0, 2^31), shift in [1, 62], |bias| < 2^30
 * and |res_mult| < 2^15 (outside that range the output is unspecified but
 * no memory outside the output tensor is touched).  bias may be NULL (0).
 * out_bits in {2, 3, 4, 6, 8}; output codes are unsigned.  The arrays (and
 * res_mult below) must be 16-byte aligned. */
typedef struct {
  const int32_t *mult;
  const int32_t *shift;
  const int32_t *bias;
  int32_t out_bits;
} palq_requant;

/* Shortcut added to t in int64 before requantisation, at the DESTINATION
 * channel of the cyclic permutation.  At most one of the two kinds:
 *  - identity: t += res_mult[c] * identity[pixel, dest channel], where
 *    `identity` has the output's shape (any unsigned bits) and res_mult is
 *    indexed like the requant arrays (device, groups*cout_pg int32);
 *  - projection: t += the int32 accumulator, at the destination channel, of
 *    the 1x1 grouped convolution of proj_in with proj_w at stride
 *    proj_stride, pad 0 (proj_w: same groups and cout_pg as the main filter,
 *    kh = kw = 1; proj_in: unsigned codes, groups = proj_w->groups). */
typedef struct {
  const palq_act *identity;
  const int32_t *res_mult;
  const palq_act *proj_in;
  const palq_filter *proj_w;
  int32_t proj_stride;
} palq_residual;

/* ---------------------------------------------------------------- context */

/* Creates a context on HIP device `device` (or -1: validate only) that
 * enqueues on `hip_stream` (a hipStream_t; NULL = the null stream).
 * Returns PALQ_ERR_DEVICE when the device cannot be used. */
palq_status palq_create(int32_t device, void *hip_stream, palq_ctx **out);
void palq_destroy(palq_ctx *ctx);
/* Later calls enqueue on hip_stream.  The new stream first waits for the
 * work already queued on the old one (which may still read context memory
 * that later calls reuse). */
palq_status palq_set_stream(palq_ctx *ctx, void *hip_stream);
/* Matrix-core format of 2-, 3- and 4-bit grouped convolutions (Section 4.1):
 * with enable = 1 (the default; environment PALQ_CONV_FP4=0 starts a context
 * at 0) a layer whose filter, outputs and shortcut have its inputs' width and
 * whose accumulator bound sum |w| |x| stays below 2^23 runs on the FP4 (E2M1)
 * matrix cores if it is a 2-bit layer, on the FP6 (E2M3) ones if it is a 3- or
 * 4-bit layer, any channel count, where its fp32 accumulator is exact; with 0
 * every layer runs on int8.  Results are identical either way.  Applies to
 * palq_group_conv calls and networks created after the call.
 * PALQ_ERR_ARG: enable not 0 or 1. */
palq_status palq_set_conv_fp4(palq_ctx *ctx, int32_t enable);
/* Execution of wide grouped convolutions as the bit-level decomposition of
 * Section 3.2 (Eq. 4), the baseline PalQuant is set against (Section 5.2,
 * Table 2): with enable = 1 a layer with unsigned M-bit inputs, M-bit
 * weights and M-bit outputs, M in {4, 6, 8}, 64-channel blocks and an
 * optional M-bit identity or projection shortcut splits every code into
 * M / 2 2-bit chunks and runs the (M / 2)^2 chunk products of each MAC on
 * the FP4 matrix cores, shifted by 4^(i+j) and summed exactly
 * ("conv_bitdecomp_kernel"), where the accumulator bounds allow it; with 0
 * (the default) such layers run directly on int8.  Results are identical
 * either way.  Applies to palq_group_conv calls and networks created after
 * the call.  PALQ_ERR_ARG: enable not 0 or 1. */
palq_status palq_set_conv_bitdecomp(palq_ctx *ctx, int32_t enable);
/* Waits for all work on the context's stream; reports deferred device errors. */
palq_status palq_sync(palq_ctx *ctx);
/* Reason for the last failed call on ctx; owned by ctx, valid until its next call. */
const char *palq_last_error(const palq_ctx *ctx);
/* Library build string (host; static storage). */
const char *palq_version(void);

/* Bytes of one packed row of `codes` codes at `bits` bits (-1 if invalid). */
int64_t palq_row_bytes(int32_t codes, int32_t bits);
/* Bytes of a packed activation tensor (-1 if the descriptor is invalid). */
int64_t palq_act_bytes(const palq_act *a);

/* ------------------------------------------------------------ data layout */

/* Packs one code per byte, [n][h][w][groups*ch_per_group] (int8 for signed,
 * uint8 for unsigned codes), into `out`'s layout.  Codes outside the b-bit
 * range are truncated to their low b bits. */
palq_status palq_pack(palq_ctx *ctx, const void *codes, const palq_act *out);
/* The inverse: one code per byte, signed codes sign-extended. */
palq_status palq_unpack(palq_ctx *ctx, const palq_act *in, void *codes);

/* ------------------------------------------------------------ hot path */

/* Uniform quantiser, Section 3.2 Eq. 2, elementwise over an fp32 NHWC tensor
 * x of out's shape: d = x - l, r = u - l, t = d / r (IEEE fp32, correctly
 * rounded), t = min(t, 1), t = (t >= 0 ? t : 0) (NaN -> 0),
 * q = rint(t * (2^b - 1)) with ties to even, and q - 2^(b-1) for signed
 * codes.  If l or u is NaN both are taken as the min and max of the non-NaN
 * elements of x (computed on the device); range_out (device, 2 floats,
 * nullable) receives the l and u used.  Host check: u > l and u - l finite
 * when both are given.  If the calibrated range is empty or degenerate the
 * output is all zero codes (the minimum code when signed). */
palq_status palq_quantize(palq_ctx *ctx, const float *x, float l, float u, const palq_act *out,
                          float *range_out);

/* One PalQuant layer: G parallel B-bit convolutions (Section 4.1; Eq. 1 per
 * group), int32 accumulation, then requantisation (palq_requant) with the
 * optional shortcut (palq_residual), and the cyclic permutation of Eq. 8
 * applied `shuffle_steps` times as the write address: the result of source
 * group g is stored in group (g + shuffle_steps) mod G.
 *   in  : unsigned codes of 2, 3, 4, 6 or 8 bits, or signed 8-bit codes;
 *         groups == w->groups, ch_per_group == w->cin_pg
 *   out : n x ho x wo, groups == w->groups, ch_per_group == w->cout_pg,
 *         bits == rq->out_bits, unsigned; ho = (h + 2 pad - kh)/stride + 1
 *   acc_dump (nullable, 16-byte aligned): int32 [n][ho][wo][groups*cout_pg], the sum of all
 *         products that land in each output channel (destination order:
 *         the permuted main accumulator plus any projection accumulator).
 * PALQ_ERR_OVERFLOW when K*max|code|*max|weight| (K = kh*kw*cin_pg), plus
 * the same bound of the projection product, reaches 2^26 for 2-bit inputs
 * or 2^30 for wider ones; a projection input is unsigned codes.  out
 * must not
 * overlap any input.  Every call prepacks the filter again, into context
 * memory that it grows (allocating) when a call needs more than any before;
 * it never synchronises.  A graph that captured the call may hold that memory,
 * which a later, larger call frees: capture palq_group_conv_noalloc or a plan
 * instead.  A loop over one layer plans it once
 * (palq_conv_plan_create) and runs the plan (palq_conv_run). */
palq_status palq_group_conv(palq_ctx *ctx, const palq_act *in, const palq_filter *w, int32_t stride,
                            int32_t pad, const palq_requant *rq, const palq_residual *res,
                            int32_t shuffle_steps, const palq_act *out, int32_t *acc_dump);

/* palq_group_conv for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, checks, arithmetic and results as
 * palq_group_conv, but the layer's prepacked filter and requant constants go
 * into a static device buffer of PALQ_NOALLOC_SCRATCH_BYTES that the library
 * holds on every GPU it runs on (until the process ends) instead of context
 * memory, and the call allocates, frees and synchronises nothing.  Every
 * call on one GPU shares that buffer and it keeps the last call's contents:
 * calls on one stream are ordered, calls that overlap on one GPU (other
 * streams, contexts or host threads) race.  PALQ_ERR_UNSUPPORTED (nothing
 * written) when the prepacked filter and constants of the layer exceed the
 * buffer; PALQ_ERR_DEVICE when the buffer is unavailable on this device. */
#define PALQ_NOALLOC_SCRATCH_BYTES (16 << 20)
palq_status palq_group_conv_noalloc(palq_ctx *ctx, const palq_act *in, const palq_filter *w, int32_t stride,
                                    int32_t pad, const palq_requant *rq, const palq_residual *res,
                                    int32_t shuffle_steps, const palq_act *out, int32_t *acc_dump);

/* A planned layer: the filter, the requant and shortcut parameters of one
 * palq_group_conv layer, prepacked into the matrix-core operand order with
 * its requant constants and its kernel chosen, once, for repeated runs. */
typedef struct palq_conv_plan palq_conv_plan;

/* Plans the layer palq_group_conv computes (same arguments and checks,
 * Section 4.1 / Eq. 1 per group, Eq. 8 as the write address): copies w,
 * rq's arrays, res->res_mult and res->proj_w into device memory the plan
 * owns, prepacks the filter, computes the requant constants and reads back
 * which epilogue applies (this call synchronises the context's stream once).
 * Only the shapes, bits, signs and layouts of in, out, res->identity and res->proj_in
 * are used; their data pointers are ignored.  The caller may free the
 * parameter arrays once this returns.  A validate-only context returns a
 * plan that runs nothing.  Errors as palq_group_conv; PALQ_ERR_NOMEM. */
palq_status palq_conv_plan_create(palq_ctx *ctx, const palq_act *in, const palq_filter *w, int32_t stride,
                                  int32_t pad, const palq_requant *rq, const palq_residual *res,
                                  int32_t shuffle_steps, const palq_act *out, palq_conv_plan **plan);
/* Runs a plan on device tensors of the planned shapes: in, out, res_in (the
 * identity shortcut's codes or the projection input, as planned; NULL when
 * the plan has no shortcut) and acc_dump (nullable; as in palq_group_conv),
 * all 16-byte aligned.  Enqueues the planned kernels on the context's
 * stream and nothing else: no allocation, no synchronisation, no host copy,
 * so it may be captured into a HIP graph.  PALQ_ERR_ARG for a plan of
 * another context, null, misaligned or overlapping pointers, or a shortcut
 * input that does not match the plan. */
palq_status palq_conv_run(palq_ctx *ctx, const palq_conv_plan *plan, const void *in, const void *res_in, void *out,
                          int32_t *acc_dump);
/* Frees a plan (waits for device work that still reads it). */
void palq_conv_plan_destroy(palq_conv_plan *plan);
/* The kernel family a plan runs without an accumulator dump (static host
 * string, e.g. "conv_fp4_kernel"; with "[wide]" where the requant
 * parameters need that build; "" for a validate-only plan; NULL for a null
 * plan). */
const char *palq_conv_plan_kernels(const palq_conv_plan *plan);

/* The cyclic permutation of Section 4.2 (Eq. 6-8) on its own:
 * out[pixel, (g + steps) mod G, :] = in[pixel, g, :], any integer steps.
 * in and out have the same shape and bits and must not overlap. */
palq_status palq_cyclic_shuffle(palq_ctx *ctx, const palq_act *in, int32_t steps,
                                const palq_act *out);

/* The cyclic shuffle module of Section 4.2 (Eq. 9-10), Z = X + Conv1x1(Y)
 * with Y = CyclicPermute(X) (Eq. 8, one step), as an integer layer:
 *   t[p, j, k] = sum_c w[j][k][c] * in[p, (j - 1) mod G, c] + bias[j*C + k]
 *                + res_mult[j*C + k] * in[p, j, k]
 *   out[p, j, k] = clamp(floor((t M + 2^(sh-1)) / 2^sh), 0, 2^out_bits - 1)
 * with M, sh = rq->mult, rq->shift [j*C + k].  Every per-channel array is
 * indexed by the module's output channel j*C + k.
 *   in  : unsigned codes of 2, 3 or 4 bits, G groups of C codes
 *   w   : 1x1 filter, groups G, cout_pg == cin_pg == C, bits == in bits
 *   out : in's n, h, w, groups and C; bits == rq->out_bits (2, 3, 4 or 8)
 *   res_mult: device int32 [G*C], |res_mult| < 2^15
 * Device pointers, caller-owned; out must not overlap in.  Runs as one
 * grouped 1x1 layer that stores its branch one group on with the identity
 * shortcut from in, its per-group parameters rotated by one group into
 * context-owned memory first (asynchronously, on the context stream).
 * Errors as palq_group_conv. */
palq_status palq_shuffle_module(palq_ctx *ctx, const palq_act *in, const palq_filter *w,
                                const palq_requant *rq, const int32_t *res_mult, const palq_act *out);

/* Channel shuffle across the groups of each pixel (the per-stage channel
 * shuffle of Section 4.3 and Table 3; the [G][C] channel matrix transposed
 * to [C][G]): out channel o = g*C + c takes in channel (o mod G)*C + o / G.
 * in and out have the same shape and bits and must not overlap. */
palq_status palq_channel_shuffle(palq_ctx *ctx, const palq_act *in, const palq_act *out);

/* k x k max pool with stride and zero-area padding (max over the in-image
 * part of each window) on unsigned codes; out has in's groups and bits. */
palq_status palq_maxpool(palq_ctx *ctx, const palq_act *in, int32_t k, int32_t stride, int32_t pad,
                         const palq_act *out);

/* Global average pool kept as the exact integer sum over h x w of unsigned
 * codes: out int32 [n][groups*ch_per_group]. */
palq_status palq_avgsum(palq_ctx *ctx, const palq_act *in, int32_t *out);

/* Fully connected layer on integer features (Eq. 1):
 * logits[i][o] = sum_c x[i][c] * w[o][c], x int32 [n][cin], w int8
 * [cout][cin], logits int32 [n][cout].  The sum is formed modulo 2^32, so a
 * logit is exact whenever its true value fits int32. */
palq_status palq_fc(palq_ctx *ctx, const int32_t *x, int32_t n, int32_t cin, const int8_t *w,
                    int32_t cout, int32_t *logits);

/* ------------------------------------------------------------ networks */

#define PALQ_OP_CONV 1
#define PALQ_OP_MAXPOOL 2
#define PALQ_OP_AVGSUM 3
#define PALQ_OP_FC 4
#define PALQ_OP_SHUFFLE_MODULE 5
#define PALQ_OP_CHANNEL_SHUFFLE 6

#define PALQ_NET_KEEP_ALL 1 /* every tensor keeps its own buffer (for inspection) */
#define PALQ_NET_TIMING 2   /* record a HIP event pair around every layer      */
#define PALQ_NET_GRAPH 4    /* replay forwards from a captured HIP graph: the
                             * first forward runs eagerly, later ones capture
                             * the launch sequence once per (input, logits, l,
                             * u, stream) and replay it; input contents may
                             * change between calls.  Not with PALQ_NET_TIMING. */
#define PALQ_NET_PIXEL_LAYOUT 8 /* keep every tensor in PALQ_LAYOUT_PIXEL; by
                                 * default a conv, channel shuffle or max pool
                                 * output of several groups whose every reader
                                 * takes it with those groups is stored in
                                 * PALQ_LAYOUT_GROUP (palq_net_tensor reports
                                 * each tensor's layout) */

/* One layer of a network.  Tensor ids: 0 is the network input; each layer
 * writes a new id `dst` larger than every id before it.  Every pointer in
 * a layer is a host or device pointer (any address HIP's default copy kind
 * accepts) to data that palq_net_create copies into the network's own pool
 * before it returns (the caller may free it afterwards):
 *   w.data / proj_w.data: packed filter bytes; mult/shift/bias/res_mult:
 *   int32 [groups*cout_pg]; fc_w: int8 [fc_out][cin].
 *  PALQ_OP_CONV    src (codes, viewed as w.groups rows of w.cin_pg codes; a
 *                  tensor may be re-grouped when its rows have no padding),
 *                  w, stride, pad, mult/shift/bias (bias nullable), out_bits,
 *                  shuffle_steps; optional identity shortcut res_src (>= 0)
 *                  with res_mult, or projection proj_src (>= 0) with proj_w
 *                  and proj_stride.  Same arithmetic as palq_group_conv.
 *  PALQ_OP_SHUFFLE_MODULE src, w (1x1, cout_pg == cin_pg), mult/shift/bias
 *                  (bias nullable), out_bits, res_mult: the cyclic shuffle
 *                  module of palq_shuffle_module (the other conv fields are
 *                  ignored).
 *  PALQ_OP_CHANNEL_SHUFFLE src -> the same shape (palq_channel_shuffle).
 *  PALQ_OP_MAXPOOL src, pool_k, pool_stride, pool_pad.
 *  PALQ_OP_AVGSUM  src -> int32 sums [n][channels].
 *  PALQ_OP_FC      src (an AVGSUM output), fc_w, fc_out -> int32 logits.
 * The last layer must be PALQ_OP_FC; its output is forward's logits. */
typedef struct {
  int32_t op;
  int32_t src, dst;
  palq_filter w;
  int32_t stride, pad;
  const int32_t *mult, *shift, *bias;
  int32_t out_bits;
  int32_t shuffle_steps;
  int32_t res_src;
  const int32_t *res_mult;
  int32_t proj_src;
  palq_filter proj_w;
  int32_t proj_stride;
  int32_t pool_k, pool_stride, pool_pad;
  const int8_t *fc_w;
  int32_t fc_out;
} palq_layer;

/* Validates the layer list against the input descriptor (shape, bits, sign;
 * its data pointer is ignored), plans buffers, copies all parameters to the
 * device and returns a network bound to ctx.  flags: PALQ_NET_*. */
palq_status palq_net_create(palq_ctx *ctx, const palq_act *input, const palq_layer *layers,
                            int32_t n_layers, int32_t flags, palq_net **out);
void palq_net_destroy(palq_net *net);

/* Runs the network on `input` (device, packed as the input descriptor says)
 * and writes logits (device, int32 [n][fc_out]).  Asynchronous. */
palq_status palq_forward(palq_ctx *ctx, palq_net *net, const void *input, int32_t *logits);

/* The quantiser of Section 3.2 Eq. 2 (as palq_quantize with fixed l, u and
 * signed 8-bit codes) followed by palq_forward, for a network whose input
 * descriptor is a signed 8-bit image with one group of 3 channels.  x:
 * device fp32 [n][h][w][3] of that shape, 4-byte aligned.  Results are
 * identical to palq_quantize into an input tensor and palq_forward on it;
 * where the first layer copies its input with a zero border the codes are
 * written straight into that copy (no separate input tensor or copy).
 * Errors: PALQ_ERR_ARG for another input format, null or misaligned
 * pointers, or l, u not finite with u > l.  Asynchronous. */
palq_status palq_forward_image(palq_ctx *ctx, palq_net *net, const float *x, float l, float u, int32_t *logits);

/* Descriptor (with device data pointer) of tensor `id` after a forward pass.
 * Conv/maxpool outputs are packed codes in the layout the descriptor names
 * (see PALQ_NET_PIXEL_LAYOUT; palq_unpack reads either); an AVGSUM output
 * is reported with bits = 32 (int32 values, one per channel, h = w = 1).
 * Valid for every id only with PALQ_NET_KEEP_ALL; otherwise buffers are
 * reused between layers. */
palq_status palq_net_tensor(const palq_net *net, int32_t id, palq_act *desc);

/* Algorithmic work of one forward pass: 2 * multiply-accumulates of every
 * conv (main and projection) and FC layer (host). */
int64_t palq_net_ops(const palq_net *net);

/* The kernels a forward pass launches for layer `layer`, as the library's
 * own selection rules pick them at create time (host string owned by net,
 * valid until palq_net_destroy): e.g. "conv_fp4_kernel" or
 * "quantize_pad4_kernel + stem_pool_kernel"; "" for a layer that an earlier
 * layer's launch already covers (a max pool fused into the stem) and for
 * every layer of a validate-only network.  image = 0: palq_forward,
 * 1: palq_forward_image; layer = -1 names forward_image's quantiser pass
 * into a buffer of its own ("" when the codes go straight into the stem's
 * zero-border input).  NULL for a null net, a bad index or image. */
const char *palq_net_layer_kernels(const palq_net *net, int32_t layer, int32_t image);

/* With PALQ_NET_TIMING: per-layer device time of every forward since the
 * last reset, summed, in milliseconds (host array of n_layers floats), and
 * the number of forwards it covers.  Synchronises the stream. */
palq_status palq_net_layer_times(palq_net *net, float *ms, int32_t *forwards);
palq_status palq_net_reset_times(palq_net *net);

/* ------------------------------------------- 8-bit transformer operators
 *
 * The products and the attention of a transformer whose weights,
 * activations and key/value cache are 8-bit codes: what a language or vision
 * model served beside the convolutional networks above needs.  Floating
 * tensors are fp32, fp16 or bf16; codes are int8 with fp32 scales.
 *
 * Quantiser of these operators, in fp32 arithmetic, over a row (one token) or
 * a block (the tokens of one cache page, one head):
 *   a = max |x|;  s = max(a * fl(1/127), 2^-100);
 *   code = clamp(rint(x * fl(1/s)), -127, 127), ties to even.
 * A row, or new tokens of a block, with an element that is not finite give
 * scale NaN and codes 0, so the results that depend on them, and no others,
 * are NaN.  A block keeps a NaN until its page starts afresh.
 */
#define PALQ_F32 0
#define PALQ_F16 1
#define PALQ_BF16 2
#define PALQ_I8 3 /* codes, with their scales in an argument of their own */

/* Token quantiser: codes[r][0..cols) and scales[r] of each of `rows` rows of
 * x (type PALQ_F32, F16 or BF16; rows x_ld elements apart, codes codes_ld
 * bytes apart).  Pointers aligned to their elements; rows and pointers that
 * are multiples of 16 bytes apart run faster.  x, codes and scales must not
 * overlap. */
palq_status palq_quantize_rows(palq_ctx *ctx, const void *x, int32_t type, int64_t rows, int32_t cols, int64_t x_ld,
                               int8_t *codes, int64_t codes_ld, float *scales);

/* Weights of y = x W^T + bias laid out for the matrix cores, once. */
typedef struct palq_linear palq_linear;

/* w: int8 codes [n_out] rows of n_in, w_ld bytes apart, w_scale fp32 [n_out],
 * bias fp32 [n_out] or NULL; all device, copied (the caller may free them
 * once this returns; it synchronises the context's stream).  Runs of up to
 * max_rows rows need no further memory: the workspace for them (shared by all
 * products and attention calls of the context) is reserved here.
 * PALQ_ERR_OVERFLOW when n_in >= 2^17 (the int32 sum of products could
 * overflow); PALQ_ERR_NOMEM.  A validate-only context returns a layer that
 * runs nothing. */
palq_status palq_linear_create(palq_ctx *ctx, const int8_t *w, int64_t w_ld, const float *w_scale, const float *bias,
                               int32_t n_out, int32_t n_in, int64_t max_rows, palq_linear **out);
/* y[m][n] = (sum_k c[m][k] w[n][k]) * s[m] * w_scale[n] + bias[n], the sum
 * exact in int32, the rest in fp32, one rounding to y_type.  x_type PALQ_F32,
 * F16 or BF16: c, s are x's rows through the quantiser above (x_scale NULL);
 * PALQ_I8: x holds c and x_scale (device, fp32 [rows]) s.  Rows of x and y
 * are x_ld and y_ld elements apart.  Enqueues kernels only (no allocation, no
 * synchronisation): may be captured into a graph, which holds the layer's
 * and the context's memory.  PALQ_ERR_ARG: rows > max_rows, a layer of
 * another context, misaligned or overlapping (address ranges of) x and y. */
palq_status palq_linear_run(palq_ctx *ctx, const palq_linear *lin, const void *x, int32_t x_type, int64_t x_ld,
                            const float *x_scale, int64_t rows, void *y, int32_t y_type, int64_t y_ld);
/* Frees a layer (waits for device work that still reads it). */
void palq_linear_destroy(palq_linear *lin);
/* The kernel a run of `rows` floating rows takes (static host string; "" for
 * a validate-only layer, NULL for a null one). */
const char *palq_linear_kernels(const palq_linear *lin, int64_t rows);

/* A paged key/value cache of one layer.  A page holds page_tokens (16, 32, 64
 * or 128) tokens of every head, head_dim 64, 96, 128 or 256:
 *   k int8 [pages][heads][page_tokens][head_dim]
 *   v int8 [pages][heads][head_dim][page_tokens]   (channel by channel)
 *   k_scale, v_scale fp32 [pages][heads]: one scale for each block
 * all device, owned by the caller, k and v 16-byte aligned. */
typedef struct {
  int32_t pages, page_tokens, heads, head_dim;
  int8_t *k, *v;
  float *k_scale, *v_scale;
} palq_cache;

/* A batch of requests of different lengths (device arrays, host sizes).
 * Request r's token j lies on page table[r][j / page_tokens], place
 * j % page_tokens; it has lens[r] tokens.  Rows starts[r] .. starts[r + 1] of
 * the tensors of a call (`tokens` rows in all) are its LAST positions,
 * lens[r] - (starts[r + 1] - starts[r]) and on: for an append or the attention
 * of the same step, lens counts the new tokens.
 *   table int32 [requests][max_pages], lens int32 [requests],
 *   starts int32 [requests + 1]
 *   max_new: at least every request's rows; max_len: at least every lens[r]
 *   (they size the launches; closer bounds run faster).
 * Device values outside these bounds never lead outside the tensors: rows
 * past max_new and tokens past max_len, the table or 2^31 - 1024 are left out, as are
 * tokens on a page number outside [0, pages).  What is left out does not move
 * the rest: a row's position follows from lens and starts as they are. */
typedef struct {
  int32_t requests, max_pages;
  const int32_t *table, *lens, *starts;
  int64_t tokens;
  int32_t max_new, max_len;
} palq_batch;

/* Quantises the new keys and values of a batch into their pages: k, v of
 * `type`, [tokens][heads][head_dim] with rows k_row / v_row and heads k_head /
 * v_head elements apart (a head's channels are consecutive).  In a block that
 * already holds tokens the scale becomes the larger of its own and the new
 * tokens'; where it grew, old codes are rescaled to
 * rint(code * fl(s_old / s)).  A block whose first token is new starts
 * afresh, whatever its page held.  Pages of different requests must be
 * distinct where they are written.  Appending the same values again leaves
 * the cache as it is. */
palq_status palq_cache_append(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, const void *k, int64_t k_row,
                              int64_t k_head, const void *v, int64_t v_row, int64_t v_head, int32_t type);
/* The inverse: code * scale of each request's last tokens, to tensors laid
 * out as in palq_cache_append; 0 for tokens on pages out of range.  Rows that
 * are left out, or whose position is none of the request's (before 0, or past
 * max_len or the table), stay as they are.  Tensors that a call writes have no
 * two rows over each other and none over the cache; k and v may be parts of
 * one fused tensor. */
palq_status palq_cache_read(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, void *k, int64_t k_row,
                            int64_t k_head, void *v, int64_t v_row, int64_t v_head, int32_t type);

/* Attention of a batch's rows over its cached tokens.  q, out: PALQ_F16 or
 * PALQ_BF16 [tokens][q_heads][head_dim], strides in elements as above;
 * q_heads a multiple of cache->heads, query head i reads cache head
 * i / (q_heads / heads).
 *   out = sum_j p_j v_j,  p = softmax_j(scale * q . k_j)
 * over the tokens j < lens[r] that a row sees: with causal = 1 those up to its
 * own position, with window > 0 only the last `window` of them; with
 * causal = 0 all (cross attention to cached encoder states: the rows then
 * have no position, and may outnumber the tokens).  A row that sees no token
 * gives 0; rows past max_new stay as they are.  Scores, softmax and sums are
 * fp32; probabilities enter the second product in fp16: 11 bits, those below
 * 2^-14 of the row's largest with an error of 2^-25 of it.  Scales are 0 or
 * more, or NaN; blocks of any v_scale mix (0: the tokens count with the value
 * 0), but one below 2^-20 of the largest among its 64 tokens (from a multiple
 * of 64 on), or below 2^-72 of the largest of all, is rounded as if it had
 * that scale.  Long caches of few rows are split and joined in the
 * context's workspace, which may grow (never while a graph is captured:
 * PALQ_ERR_NOMEM then; run the shape once before).  out and q (address ranges)
 * must not overlap. */
palq_status palq_attention(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, const void *q, int64_t q_row,
                           int64_t q_head, int32_t q_heads, void *out, int64_t out_row, int64_t out_head, int32_t type,
                           float scale, int32_t causal, int32_t window);

/* ------------------------------------- a generation step around the cache
 *
 * What stands between the products above, the cache and the next token: norms and
 * rotation of queries and keys, attention that keeps a request's first tokens
 * beside a window or follows a tree of drafted tokens, and the log probabilities
 * by which tokens are chosen and drafts are checked.
 */

/* A batch's new tokens as trees, one a request (checking several drafts at
 * once).  mask (device, 8-byte aligned): uint64 [tokens][words], words 1 to
 * PALQ_TREE_WORDS; bit b (of word b / 64, from the lowest) of a row stands for
 * new token b of its request (row starts[r] + b) and says whether the row sees
 * it; a row's own bit is no different.  Bits past the request's new tokens are
 * ignored, new tokens past 64 words are seen by none.  The position of a row is
 * that of the request's first new token plus the number of new tokens that it
 * sees besides itself: its depth, where bits are a token's ancestors. */
#define PALQ_TREE_WORDS 16
typedef struct {
  const uint64_t *mask;
  int32_t words;
} palq_tree;

/* The frequencies of a rotation, for any number of calls. */
typedef struct palq_rotation palq_rotation;

/* freq: HOST array of `pairs` (1 to 128) finite frequencies in radians a
 * position; copied.  Pair i of a head is channels i and i + pairs, or 2 i and
 * 2 i + 1 with interleaved = 1; channels from 2 pairs on do not rotate.
 * Synchronises the context's stream.  PALQ_ERR_NOMEM.  A validate-only context
 * returns a rotation that runs nothing. */
palq_status palq_rotation_create(palq_ctx *ctx, const double *freq, int32_t pairs, int32_t interleaved, palq_rotation **out);
/* Frees a rotation (waits for device work that still reads it). */
void palq_rotation_destroy(palq_rotation *rot);

/* Queries or keys of a batch and where their results go: [tokens][heads][head_dim], strides
 * in elements as in palq_cache_append; weight: fp32 [head_dim], or NULL for ones. */
typedef struct {
  const void *x;
  int64_t row, head;
  void *out;
  int64_t out_row, out_head;
  const float *weight;
  int32_t heads;
} palq_heads;

/* RMS norm of every head of queries and keys, then the rotation of its pairs
 * (a, b) by position, in fp32 and with one rounding:
 *   y = x / sqrt(mean(x^2) + eps) * weight,  t = position * freq,
 *   (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t)
 * q, k (either may be NULL): `type` (PALQ_F32, F16 or BF16), head_dim 64, 96, 128
 * or 256.  eps 0: no norm, and no weights; else a normal number.  rot NULL: no
 * rotation.  Row i of request r is at position lens[r] - starts[r + 1] + i, or where `tree`
 * (nullable) puts it; its fraction of a turn is that of position * freq, freq as given,
 * to position 2^-65, however far the position.  Of the batch, table, max_pages and
 * max_len have no effect.  Rows past max_new stay as they are.  Results may be
 * in place (the same pointer and strides); other overlaps of a result are
 * refused, where tensors of different strides count as their whole ranges.
 * Enqueues one kernel (or more where bounds are loose), and nothing else. */
palq_status palq_norm_rotate(palq_ctx *ctx, const palq_rotation *rot, const palq_batch *batch, const palq_tree *tree,
                             const palq_heads *q, const palq_heads *k, int32_t head_dim, int32_t type, float eps);

/* palq_attention (causal) where a window leaves a request's first tokens
 * visible: a row at position p sees the tokens j <= p with j > p - window or
 * j < sinks.  window 0: all of them, whatever sinks.  What lies between is not
 * read.  Arguments, arithmetic, workspace and errors as palq_attention. */
palq_status palq_attention_sinks(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, const void *q, int64_t q_row,
                                 int64_t q_head, int32_t q_heads, void *out, int64_t out_row, int64_t out_head, int32_t type,
                                 float scale, int32_t window, int32_t sinks);

/* palq_attention of drafted tokens that form a tree, appended to the cache in
 * any order of their rows: a row sees the tokens before the request's first new
 * one (with a window those that palq_attention_sinks leaves at the row's position in the
 * tree), and of the new ones those whose bit its mask has, whatever the window.
 * A row that sees none gives 0.  Once a branch is accepted, appending its tokens
 * again with lens shortened to it puts them in order. */
palq_status palq_attention_tree(palq_ctx *ctx, const palq_cache *cache, const palq_batch *batch, const palq_tree *tree, const void *q,
                                int64_t q_row, int64_t q_head, int32_t q_heads, void *out, int64_t out_row, int64_t out_head,
                                int32_t type, float scale, int32_t window, int32_t sinks);

/* Log probabilities of given tokens, entropy, and the most probable tokens:
 *   l[r][i] = scale x[r][i] - ln sum_j exp(scale x[r][j])   (natural logarithm)
 * logits x: `type` (PALQ_F32, F16 or BF16) [rows], ld elements apart, of `vocab`
 * (up to 2^30) tokens; scale (one over a temperature): 2^-119 to 2^119.
 *   ids int32 [rows][given] -> out fp32 [rows][given]: l of those tokens (NaN
 *   for an id outside [0, vocab)); given may be 0
 *   entropy fp32 [rows] (nullable): -sum_i exp(l) l
 *   top_ids int32 [rows][top], top_out fp32 [rows][top]: the `top` (0 to
 *   PALQ_TOP_MAX, at most vocab) largest logits in order, of equal ones the
 *   lowest index first (-0 equals 0), and their l
 * all device.  A token of logit -inf has l = -inf and counts 0 in the entropy; a
 * row of nothing else has l = -inf throughout and entropy 0.  A row with NaN or
 * +inf has NaN for every l and its entropy, and -1 for its top ids.  Sums are fp32
 * under the row's largest logit.  Few rows are split and joined in the context's
 * workspace, which may grow (never while a graph is captured: PALQ_ERR_NOMEM
 * then; run the shape once before); where a row is cut moves l and the entropy by
 * their rounding, the list not at all.  Graphs that hold calls of one context, these or
 * attention's, share its workspace: they are replayed one after the other. */
#define PALQ_TOP_MAX 64
palq_status palq_log_probs(palq_ctx *ctx, const void *logits, int32_t type, int64_t rows, int32_t vocab, int64_t ld, float scale,
                           const int32_t *ids, int32_t given, float *out, float *entropy, int32_t top, int32_t *top_ids, float *top_out);

#ifdef __cplusplus
}
#endif
#endif /* PALQ_H */
