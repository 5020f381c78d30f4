"""ctypes binding of libpalq.so (include/palq.h).

Argument marshalling only: every step of the path runs in the HIP library.
torch supplies device memory and the stream.  Importing this module loads the
library and raises ImportError if it has not been built
(python -m paper_2208_01944_amd.build).
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpalq.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2208_01944_amd.build`")

# torch ships its own HIP runtime under the same soname (libamdhip64.so.7).
# Loading torch first makes the library bind to that runtime, so the process
# has one HIP runtime that both use (loaded the other way round, the
# library's context creation fails on the GPU machine).
import torch  # noqa: E402,F401

_lib = ctypes.CDLL(LIB_PATH)

c_i32, c_i64, c_p, c_f = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float

OK, ERR_ARG, ERR_UNSUPPORTED, ERR_OVERFLOW, ERR_DEVICE, ERR_NOMEM = 0, -1, -2, -3, -4, -5
OP_CONV, OP_MAXPOOL, OP_AVGSUM, OP_FC, OP_SHUFFLE_MODULE, OP_CHANNEL_SHUFFLE = 1, 2, 3, 4, 5, 6
NET_KEEP_ALL, NET_TIMING, NET_GRAPH, NET_PIXEL_LAYOUT = 1, 2, 4, 8
LAYOUT_PIXEL, LAYOUT_GROUP = 0, 1
F32, F16, BF16, I8 = 0, 1, 2, 3  # element types of the transformer operators
_INT_MAX = (1 << 31) - 1
_F32_MIN = 2.0 ** -126  # the smallest normal number
_F32, _I32 = torch.float32, torch.int32
_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16, torch.int8: I8}


class Act(ctypes.Structure):
    _fields_ = [("n", c_i32), ("h", c_i32), ("w", c_i32), ("groups", c_i32),
                ("ch_per_group", c_i32), ("bits", c_i32), ("is_signed", c_i32), ("layout", c_i32),
                ("data", c_p)]


class Filter(ctypes.Structure):
    _fields_ = [("groups", c_i32), ("cout_pg", c_i32), ("cin_pg", c_i32), ("kh", c_i32),
                ("kw", c_i32), ("bits", c_i32), ("data", c_p)]


class Requant(ctypes.Structure):
    _fields_ = [("mult", c_p), ("shift", c_p), ("bias", c_p), ("out_bits", c_i32)]


class Residual(ctypes.Structure):
    _fields_ = [("identity", ctypes.POINTER(Act)), ("res_mult", c_p),
                ("proj_in", ctypes.POINTER(Act)), ("proj_w", ctypes.POINTER(Filter)),
                ("proj_stride", c_i32)]


class Layer(ctypes.Structure):
    _fields_ = [("op", c_i32), ("src", c_i32), ("dst", c_i32), ("w", Filter), ("stride", c_i32),
                ("pad", c_i32), ("mult", c_p), ("shift", c_p), ("bias", c_p), ("out_bits", c_i32),
                ("shuffle_steps", c_i32), ("res_src", c_i32), ("res_mult", c_p),
                ("proj_src", c_i32), ("proj_w", Filter), ("proj_stride", c_i32),
                ("pool_k", c_i32), ("pool_stride", c_i32), ("pool_pad", c_i32), ("fc_w", c_p),
                ("fc_out", c_i32)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("pages", c_i32), ("page_tokens", c_i32), ("heads", c_i32), ("head_dim", c_i32),
                ("k", c_p), ("v", c_p), ("k_scale", c_p), ("v_scale", c_p)]


class BatchDesc(ctypes.Structure):
    _fields_ = [("requests", c_i32), ("max_pages", c_i32), ("table", c_p), ("lens", c_p), ("starts", c_p),
                ("tokens", c_i64), ("max_new", c_i32), ("max_len", c_i32)]


class HeadsDesc(ctypes.Structure):
    _fields_ = [("x", c_p), ("row", c_i64), ("head", c_i64), ("out", c_p), ("out_row", c_i64), ("out_head", c_i64), ("weight", c_p),
                ("heads", c_i32)]


_pack_heads = struct.Struct("@PqqPqqPi").pack_into  # (as HeadsDesc lies in memory)
_HEADS_SIZE = ctypes.sizeof(HeadsDesc)


class TreeDesc(ctypes.Structure):
    _fields_ = [("mask", c_p), ("words", c_i32)]


def _sig(name, res, *args):
    f = getattr(_lib, name)
    f.restype = res
    f.argtypes = list(args)
    return f


P_ACT, P_FIL = ctypes.POINTER(Act), ctypes.POINTER(Filter)
_create = _sig("palq_create", c_i32, c_i32, c_p, ctypes.POINTER(c_p))
_destroy = _sig("palq_destroy", None, c_p)
_set_stream = _sig("palq_set_stream", c_i32, c_p, c_p)
_sync = _sig("palq_sync", c_i32, c_p)
_set_conv_fp4 = _sig("palq_set_conv_fp4", c_i32, c_p, c_i32)
_set_conv_bitdecomp = _sig("palq_set_conv_bitdecomp", c_i32, c_p, c_i32)
_last_error = _sig("palq_last_error", ctypes.c_char_p, c_p)
_version = _sig("palq_version", ctypes.c_char_p)
_row_bytes = _sig("palq_row_bytes", c_i64, c_i32, c_i32)
_act_bytes = _sig("palq_act_bytes", c_i64, P_ACT)
_pack = _sig("palq_pack", c_i32, c_p, c_p, P_ACT)
_unpack = _sig("palq_unpack", c_i32, c_p, P_ACT, c_p)
_quantize = _sig("palq_quantize", c_i32, c_p, c_p, c_f, c_f, P_ACT, c_p)
_group_conv = _sig("palq_group_conv", c_i32, c_p, P_ACT, P_FIL, c_i32, c_i32,
                   ctypes.POINTER(Requant), ctypes.POINTER(Residual), c_i32, P_ACT, c_p)
_group_conv_noalloc = _sig("palq_group_conv_noalloc", c_i32, c_p, P_ACT, P_FIL, c_i32, c_i32,
                           ctypes.POINTER(Requant), ctypes.POINTER(Residual), c_i32, P_ACT, c_p)
NOALLOC_SCRATCH_BYTES = 16 << 20
_conv_plan_create = _sig("palq_conv_plan_create", c_i32, c_p, P_ACT, P_FIL, c_i32, c_i32, ctypes.POINTER(Requant),
                         ctypes.POINTER(Residual), c_i32, P_ACT, ctypes.POINTER(c_p))
_conv_run = _sig("palq_conv_run", c_i32, c_p, c_p, c_p, c_p, c_p, c_p)
_conv_plan_destroy = _sig("palq_conv_plan_destroy", None, c_p)
_conv_plan_kernels = _sig("palq_conv_plan_kernels", ctypes.c_char_p, c_p)
_shuffle = _sig("palq_cyclic_shuffle", c_i32, c_p, P_ACT, c_i32, P_ACT)
_channel_shuffle = _sig("palq_channel_shuffle", c_i32, c_p, P_ACT, P_ACT)
_shuffle_module = _sig("palq_shuffle_module", c_i32, c_p, P_ACT, P_FIL, ctypes.POINTER(Requant), c_p, P_ACT)
_maxpool = _sig("palq_maxpool", c_i32, c_p, P_ACT, c_i32, c_i32, c_i32, P_ACT)
_avgsum = _sig("palq_avgsum", c_i32, c_p, P_ACT, c_p)
_fc = _sig("palq_fc", c_i32, c_p, c_p, c_i32, c_i32, c_p, c_i32, c_p)
_net_create = _sig("palq_net_create", c_i32, c_p, P_ACT, ctypes.POINTER(Layer), c_i32, c_i32,
                   ctypes.POINTER(c_p))
_net_destroy = _sig("palq_net_destroy", None, c_p)
_forward = _sig("palq_forward", c_i32, c_p, c_p, c_p, c_p)
_forward_image = _sig("palq_forward_image", c_i32, c_p, c_p, c_p, c_f, c_f, c_p)
_net_tensor = _sig("palq_net_tensor", c_i32, c_p, c_i32, P_ACT)
_net_ops = _sig("palq_net_ops", c_i64, c_p)
_net_layer_kernels = _sig("palq_net_layer_kernels", ctypes.c_char_p, c_p, c_i32, c_i32)
_net_layer_times = _sig("palq_net_layer_times", c_i32, c_p, ctypes.POINTER(c_f), ctypes.POINTER(c_i32))
_net_reset_times = _sig("palq_net_reset_times", c_i32, c_p)
_quantize_rows = _sig("palq_quantize_rows", c_i32, c_p, c_p, c_i32, c_i64, c_i32, c_i64, c_p, c_i64, c_p)
_linear_create = _sig("palq_linear_create", c_i32, c_p, c_p, c_i64, c_p, c_p, c_i32, c_i32, c_i64, ctypes.POINTER(c_p))
_linear_run = _sig("palq_linear_run", c_i32, c_p, c_p, c_p, c_i32, c_i64, c_p, c_i64, c_p, c_i32, c_i64)
_linear_destroy = _sig("palq_linear_destroy", None, c_p)
_linear_kernels = _sig("palq_linear_kernels", ctypes.c_char_p, c_p, c_i64)
P_CACHE, P_BATCH = ctypes.POINTER(CacheDesc), ctypes.POINTER(BatchDesc)
_cache_append = _sig("palq_cache_append", c_i32, c_p, P_CACHE, P_BATCH, c_p, c_i64, c_i64, c_p, c_i64, c_i64, c_i32)
_cache_read = _sig("palq_cache_read", c_i32, c_p, P_CACHE, P_BATCH, c_p, c_i64, c_i64, c_p, c_i64, c_i64, c_i32)
_attention = _sig("palq_attention", c_i32, c_p, P_CACHE, P_BATCH, c_p, c_i64, c_i64, c_i32, c_p, c_i64, c_i64, c_i32, c_f,
                  c_i32, c_i32)
P_TREE = ctypes.POINTER(TreeDesc)
_rotation_create = _sig("palq_rotation_create", c_i32, c_p, ctypes.POINTER(ctypes.c_double), c_i32, c_i32, ctypes.POINTER(c_p))
_rotation_destroy = _sig("palq_rotation_destroy", None, c_p)
_norm_rotate = _sig("palq_norm_rotate", c_i32, c_p, c_p, P_BATCH, P_TREE, c_p, c_p, c_i32, c_i32, c_f)
_attention_sinks = _sig("palq_attention_sinks", c_i32, c_p, P_CACHE, P_BATCH, c_p, c_i64, c_i64, c_i32, c_p, c_i64, c_i64, c_i32, c_f,
                        c_i32, c_i32)
_attention_tree = _sig("palq_attention_tree", c_i32, c_p, P_CACHE, P_BATCH, P_TREE, c_p, c_i64, c_i64, c_i32, c_p, c_i64, c_i64, c_i32,
                       c_f, c_i32, c_i32)
_log_probs = _sig("palq_log_probs", c_i32, c_p, c_p, c_i32, c_i64, c_i32, c_i64, c_f, c_p, c_i32, c_p, c_p, c_i32, c_p, c_p)

EXPORTS = ["palq_create", "palq_destroy", "palq_set_stream", "palq_set_conv_fp4", "palq_set_conv_bitdecomp", "palq_sync", "palq_last_error",
           "palq_version", "palq_row_bytes", "palq_act_bytes", "palq_pack", "palq_unpack",
           "palq_quantize", "palq_group_conv", "palq_group_conv_noalloc", "palq_conv_plan_create",
           "palq_conv_run", "palq_conv_plan_destroy", "palq_conv_plan_kernels", "palq_shuffle_module", "palq_cyclic_shuffle",
           "palq_channel_shuffle", "palq_maxpool",
           "palq_avgsum", "palq_fc", "palq_net_create", "palq_net_destroy", "palq_forward",
           "palq_forward_image", "palq_net_tensor", "palq_net_ops", "palq_net_layer_kernels", "palq_net_layer_times",
           "palq_net_reset_times", "palq_quantize_rows", "palq_linear_create", "palq_linear_run", "palq_linear_destroy",
           "palq_linear_kernels", "palq_cache_append", "palq_cache_read", "palq_attention",
           "palq_rotation_create", "palq_rotation_destroy", "palq_norm_rotate", "palq_attention_sinks",
           "palq_attention_tree", "palq_log_probs"]


class PalqError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"palq status {status}: {msg}")
        self.status = status


def row_bytes(codes: int, bits: int) -> int:
    return int(_row_bytes(codes, bits))


def version() -> str:
    return _version().decode()


def make_act(n, h, w, groups, cpg, bits, signed=False, data=0, layout=LAYOUT_PIXEL) -> Act:
    return Act(n, h, w, groups, cpg, bits, int(bool(signed)), layout, data)


def act_bytes(a: Act) -> int:
    return int(_act_bytes(ctypes.byref(a)))


def _ptr(t):
    if t is None:
        return None
    return t.data_ptr()


class Tensor:
    """A packed code tensor in device memory: a torch uint8 buffer + its Act."""

    def __init__(self, buf, act: Act):
        self.buf = buf
        self.act = act

    @property
    def shape(self):
        a = self.act
        return (a.n, a.h, a.w, a.groups * a.ch_per_group)


class Context:
    """One palq context on a device (or -1: validate only)."""

    def __init__(self, device: int = 0, stream=None):
        self.device = device
        if device >= 0:
            import torch
            self.torch = torch
            self.dev = torch.device("cuda", device)
            if stream is None:
                stream = torch.cuda.current_stream(self.dev).cuda_stream
        else:
            self.torch = None
        self.heads = (HeadsDesc * 2)()  # norm_rotate's descriptors, filled for each call
        self.heads_at = [ctypes.addressof(h) for h in self.heads]
        h = c_p()
        st = _create(device, stream or 0, ctypes.byref(h))
        if st != OK:
            raise PalqError(st, f"palq_create(device={device}) failed")
        self.h = h

    def __del__(self):
        h = getattr(self, "h", None)
        if h:
            _destroy(h)
            self.h = None

    def _check(self, st):
        if st != OK:
            raise PalqError(st, _last_error(self.h).decode())

    def last_error(self) -> str:
        return _last_error(self.h).decode()

    def sync(self):
        self._check(_sync(self.h))

    def set_stream(self, stream):
        """palq_set_stream: later calls enqueue on `stream` (a torch stream)."""
        self._check(_set_stream(self.h, stream.cuda_stream))

    def set_conv_fp4(self, enable: bool):
        """FP4 (2-bit) and FP6 (3-bit) matrix cores for exact layers (True) or
        int8 only."""
        self._check(_set_conv_fp4(self.h, int(bool(enable))))

    def set_conv_bitdecomp(self, enable: bool):
        """Wide (4/6/8-bit) layers as the Eq. 4 bit decomposition on FP4
        matrix cores (True) or directly on int8 (False, the default)."""
        self._check(_set_conv_bitdecomp(self.h, int(bool(enable))))

    # ----------------------------------------------------------- memory
    def empty_act(self, n, h, w, groups, cpg, bits, signed=False, layout=LAYOUT_PIXEL) -> Tensor:
        a = make_act(n, h, w, groups, cpg, bits, signed, layout=layout)
        nb = act_bytes(a)
        if nb < 0:
            raise PalqError(ERR_ARG, "invalid activation descriptor")
        buf = self.torch.empty(max(nb, 16), dtype=self.torch.uint8, device=self.dev)
        a.data = buf.data_ptr()
        return Tensor(buf, a)

    def upload(self, arr, dtype=None):
        t = self.torch.from_numpy(np.ascontiguousarray(arr if dtype is None else arr.astype(dtype)))
        return t.to(self.dev)

    # ----------------------------------------------------------- layout
    def pack(self, codes, groups, bits, signed=False, layout=LAYOUT_PIXEL) -> Tensor:
        """codes: numpy [n, h, w, groups*cpg] integer codes -> packed device tensor."""
        n, h, w, c = codes.shape
        out = self.empty_act(n, h, w, groups, c // groups, bits, signed, layout=layout)
        dt = np.int8 if signed else np.uint8
        src = self.upload(np.asarray(codes).astype(dt))
        self._check(_pack(self.h, src.data_ptr(), ctypes.byref(out.act)))
        return out

    def pack_filter(self, w_codes, bits) -> tuple:
        """w_codes: numpy [G, Co, kh, kw, Ci] signed codes -> (device buffer, Filter)."""
        g, co, kh, kw, ci = w_codes.shape
        t = self.pack(np.asarray(w_codes).reshape(g * co, kh, kw, ci), 1, bits, signed=True)
        f = Filter(g, co, ci, kh, kw, bits, t.act.data)
        return t, f

    def unpack(self, t: Tensor) -> np.ndarray:
        a = t.act
        n = a.n * a.h * a.w * a.groups * a.ch_per_group
        out = self.torch.empty(max(n, 1), dtype=self.torch.uint8, device=self.dev)
        self._check(_unpack(self.h, ctypes.byref(a), out.data_ptr()))
        arr = out[:n].cpu().numpy()
        arr = arr.view(np.int8) if a.is_signed else arr
        return arr.reshape(a.n, a.h, a.w, a.groups * a.ch_per_group).astype(np.int64)

    # ----------------------------------------------------------- ops
    def quantize(self, x, l, u, out: Tensor, range_out=None):
        self._check(_quantize(self.h, _ptr(x), l, u, ctypes.byref(out.act), _ptr(range_out)))

    def group_conv(self, x: Tensor, w: Filter, stride, pad, mult, shift, bias, out: Tensor,
                   shuffle=0, identity: Tensor = None, res_mult=None, proj_in: Tensor = None,
                   proj_w: Filter = None, proj_stride=1, acc_dump=None, noalloc=False):
        """palq_group_conv (noalloc: palq_group_conv_noalloc)."""
        rq = Requant(_ptr(mult), _ptr(shift), _ptr(bias), out.act.bits)
        res = None
        if identity is not None or proj_in is not None:
            res = Residual()
            if identity is not None:
                res.identity = ctypes.pointer(identity.act)
                res.res_mult = _ptr(res_mult)
            if proj_in is not None:
                res.proj_in = ctypes.pointer(proj_in.act)
                res.proj_w = ctypes.pointer(proj_w)
                res.proj_stride = proj_stride
        fn = _group_conv_noalloc if noalloc else _group_conv
        self._check(fn(self.h, ctypes.byref(x.act), ctypes.byref(w), stride, pad,
                       ctypes.byref(rq), ctypes.byref(res) if res is not None else None,
                       shuffle, ctypes.byref(out.act), _ptr(acc_dump)))

    def shuffle_module(self, x: Tensor, w: Filter, mult, shift, bias, res_mult, out: Tensor):
        rq = Requant(_ptr(mult), _ptr(shift), _ptr(bias), out.act.bits)
        self._check(_shuffle_module(self.h, ctypes.byref(x.act), ctypes.byref(w), ctypes.byref(rq),
                                    _ptr(res_mult), ctypes.byref(out.act)))

    def channel_shuffle(self, x: Tensor, out: Tensor):
        self._check(_channel_shuffle(self.h, ctypes.byref(x.act), ctypes.byref(out.act)))

    def cyclic_shuffle(self, x: Tensor, steps, out: Tensor):
        self._check(_shuffle(self.h, ctypes.byref(x.act), steps, ctypes.byref(out.act)))

    def maxpool(self, x: Tensor, k, stride, pad, out: Tensor):
        self._check(_maxpool(self.h, ctypes.byref(x.act), k, stride, pad, ctypes.byref(out.act)))

    def avgsum(self, x: Tensor, out):
        self._check(_avgsum(self.h, ctypes.byref(x.act), _ptr(out)))

    def fc(self, x, n, cin, w, cout, logits):
        self._check(_fc(self.h, _ptr(x), n, cin, _ptr(w), cout, _ptr(logits)))

    # ----------------------------------------------------------- 8-bit transformer operators
    def quantize_rows(self, x, codes, scales):
        """palq_quantize_rows: x [rows, cols] floating -> codes int8 [rows, cols], scales fp32 [rows]."""
        if codes.dtype != torch.int8 or tuple(codes.shape) != tuple(x.shape):
            raise PalqError(ERR_ARG, "codes must be int8 of x's shape")
        _need(scales, torch.float32, x.shape[0], "scales")
        _on(self, x, codes, scales)
        if x.shape[1] > _INT_MAX:
            raise PalqError(ERR_UNSUPPORTED, "a row of 2^31 elements or more")
        xt, x_ld = _rows2(x)
        _, c_ld = _rows2(codes)
        self._check(_quantize_rows(self.h, x.data_ptr(), xt, x.shape[0], x.shape[1], x_ld, codes.data_ptr(), c_ld,
                                   scales.data_ptr()))

    def cache_append(self, cache: Cache, k, v, batch: Batch):
        """palq_cache_append: k, v [tokens, heads, head_dim] into the pages of their requests."""
        t, kr, kh, vr, vh = _pair3(self, k, v, batch, cache)
        st = _cache_append(self.h, cache.ref, batch.ref, k.data_ptr(), kr, kh, v.data_ptr(), vr, vh, t)
        if st:
            self._check(st)

    def cache_read(self, cache: Cache, k, v, batch: Batch):
        """palq_cache_read: the values of each request's last tokens into k, v [tokens, heads, head_dim]."""
        t, kr, kh, vr, vh = _pair3(self, k, v, batch, cache)
        st = _cache_read(self.h, cache.ref, batch.ref, k.data_ptr(), kr, kh, v.data_ptr(), vr, vh, t)
        if st:
            self._check(st)

    def attention(self, cache: Cache, q, out, batch: Batch, scale, causal=True, window=0, sinks=0, tree=None):
        """palq_attention: q, out [tokens, q_heads, head_dim].  sinks: first tokens that a window leaves visible
        (palq_attention_sinks); tree: int64 masks [tokens, words] of drafted tokens (palq_attention_tree)."""
        t, qr, qh, orow, oh = _pair3(self, q, out, batch, cache, True)
        if window < 0:
            raise PalqError(ERR_ARG, "window must be 0 or more")
        if sinks or tree is not None:
            if sinks < 0 or not causal:
                raise PalqError(ERR_ARG, "sinks must be 0 or more; sinks and trees are causal")
            window, sinks = min(window, _INT_MAX), min(sinks, _INT_MAX)
            if tree is None:
                st = _attention_sinks(self.h, cache.ref, batch.ref, q.data_ptr(), qr, qh, q.shape[1], out.data_ptr(), orow, oh, t, scale,
                                      window, sinks)
            else:
                st = _attention_tree(self.h, cache.ref, batch.ref, _tree(self, tree, q.shape[0]), q.data_ptr(), qr, qh, q.shape[1],
                                     out.data_ptr(), orow, oh, t, scale, window, sinks)
            if st:
                self._check(st)
            return
        st = _attention(self.h, cache.ref, batch.ref, q.data_ptr(), qr, qh, q.shape[1], out.data_ptr(), orow, oh, t, scale, causal,
                        min(window, _INT_MAX))
        if st:
            self._check(st)

    def norm_rotate(self, batch: Batch, q, q_out, k=None, k_out=None, q_weight=None, k_weight=None, eps=None, rotation=None, tree=None):
        """palq_norm_rotate: each head of q and k [tokens, heads, head_dim] normed (eps None: not) and rotated by position
        into q_out and k_out, which may be q and k.  tree: int64 masks [tokens, words]."""
        tokens, qn, dim = shape = q.shape
        dtype, d = q.dtype, self.device
        qr, qh, q1 = q.stride()
        qor, qoh, qo1 = q_out.stride()
        kind = _TYPES.get(dtype)
        if kind is None or q_out.dtype is not dtype:
            raise PalqError(ERR_ARG, "the tensors differ in type, or have no element type of the library")
        if q_out.shape != shape or q1 != 1 or qo1 != 1:
            raise PalqError(ERR_ARG, "tensors must be [tokens, heads, head_dim], results of their shapes, a head's channels consecutive")
        on = d < 0 or (q.get_device() == d and q_out.get_device() == d and batch.device == d)
        qw = kw = 0
        keys = None
        if k is not None and k_out is not None:
            kt, kn, kd = shape = k.shape
            kr, kh, k1 = k.stride()
            kor, koh, ko1 = k_out.stride()
            if k.dtype is not dtype or k_out.dtype is not dtype or kt != tokens or kd != dim or k_out.shape != shape or k1 != 1 or ko1 != 1:
                raise PalqError(ERR_ARG, "k and k_out must be as q, [tokens, heads, head_dim]")
            on = on and (d < 0 or (k.get_device() == d and k_out.get_device() == d))
            keys = self.heads_at[1]
        elif k is not None or k_out is not None:
            raise PalqError(ERR_ARG, "k and k_out go together")
        if q_weight is not None:
            if q_weight.dtype is not _F32 or q_weight.shape != (dim,) or not q_weight.is_contiguous():
                raise PalqError(ERR_ARG, "a weight must be head_dim contiguous values of torch.float32")
            on = on and (d < 0 or q_weight.get_device() == d)
            qw = q_weight.data_ptr()
        if k_weight is not None:
            if k_weight.dtype is not _F32 or k_weight.shape != (dim,) or not k_weight.is_contiguous():
                raise PalqError(ERR_ARG, "a weight must be head_dim contiguous values of torch.float32")
            on = on and (d < 0 or k_weight.get_device() == d)
            kw = k_weight.data_ptr()
        if not on:
            raise PalqError(ERR_ARG, f"tensors or batch are not on the context's device, cuda:{d}")
        if eps is None:
            eps = 0.0
        elif not eps >= _F32_MIN:  # (as fp32 it would be 0, which means no norm, or lose bits)
            raise PalqError(ERR_ARG, "eps must be a normal positive fp32 number (None: no norm)")
        if rotation is not None:
            if rotation.ctx is not self:
                raise PalqError(ERR_ARG, "rotation of another context")
            rotation = rotation.h
        if tree is not None:
            tree = _tree(self, tree, tokens)
        if batch.tokens != tokens:
            batch.tokens = batch.desc.tokens = tokens
        _pack_heads(self.heads, 0, q.data_ptr(), qr, qh, q_out.data_ptr(), qor, qoh, qw, qn)
        if keys:
            _pack_heads(self.heads, _HEADS_SIZE, k.data_ptr(), kr, kh, k_out.data_ptr(), kor, koh, kw, kn)
        elif kw:
            raise PalqError(ERR_ARG, "k_weight without k")
        st = _norm_rotate(self.h, rotation, batch.ref, tree, self.heads_at[0], keys, dim, kind, eps)
        if st:
            self._check(st)

    def log_probs(self, logits, ids, out, entropy=None, top_ids=None, top=None, scale=1.0):
        """palq_log_probs: log probabilities of ids int32 [rows, given] (or [rows]; None: none) under logits [rows, vocab] into
        out fp32 of ids' shape, entropy fp32 [rows], and the most probable tokens into top_ids int32 and top fp32 [rows, n]."""
        rows, vocab = logits.shape
        kind, ld = _rows2(logits)
        if vocab > _INT_MAX:
            raise PalqError(ERR_UNSUPPORTED, "a row of 2^31 elements or more")
        d = self.device
        on = d < 0 or logits.get_device() == d
        given = n = 0
        ip = op = ep = tp = lp = None
        if ids is not None:
            shape = ids.shape
            given = shape[1] if len(shape) == 2 else 1
            if out is None or shape[0] != rows or out.shape != shape:
                raise PalqError(ERR_ARG, "ids must have a row for each of the logits', and out their shape")
            if ids.dtype is not _I32 or out.dtype is not _F32 or len(shape) > 2 or not (ids.is_contiguous() and out.is_contiguous()):
                raise PalqError(ERR_ARG, "ids must be contiguous int32, out contiguous float32")
            on = on and (d < 0 or (ids.get_device() == d and out.get_device() == d))
            ip, op = ids.data_ptr(), out.data_ptr()
        if entropy is not None:
            if entropy.dtype is not _F32 or entropy.shape != (rows,) or not entropy.is_contiguous():
                raise PalqError(ERR_ARG, "entropy must be a contiguous float32 for each row")
            on = on and (d < 0 or entropy.get_device() == d)
            ep = entropy.data_ptr()
        if top is not None and top_ids is not None:
            m, n = shape = top.shape
            if m != rows or top_ids.shape != shape:
                raise PalqError(ERR_ARG, "top_ids and top must be [rows, n]")
            if top_ids.dtype is not _I32 or top.dtype is not _F32 or not (top_ids.is_contiguous() and top.is_contiguous()):
                raise PalqError(ERR_ARG, "top_ids must be contiguous int32, top contiguous float32")
            on = on and (d < 0 or (top_ids.get_device() == d and top.get_device() == d))
            tp, lp = top_ids.data_ptr(), top.data_ptr()
        elif top is not None or top_ids is not None:
            raise PalqError(ERR_ARG, "top_ids and top go together")
        if not on:
            raise PalqError(ERR_ARG, f"tensors are not on the context's device, cuda:{d}")
        st = _log_probs(self.h, logits.data_ptr(), kind, rows, vocab, ld, scale, ip, given, op, ep, n, tp, lp)
        if st:
            self._check(st)


class Rotation:
    """Frequencies of a rotation by position (palq_rotation_create): freq, in radians a position, one for each pair of
    channels (i, i + pairs), or (2 i, 2 i + 1) where interleaved; copied."""

    def __init__(self, ctx: Context, freq, interleaved=False):
        f = np.ascontiguousarray(freq, dtype=np.float64)
        if f.ndim != 1 or not 1 <= f.size <= 128:
            raise PalqError(ERR_ARG, "freq must be 1 to 128 numbers")
        self.ctx, self.pairs, self.interleaved = ctx, f.size, bool(interleaved)
        h = c_p()
        ctx._check(_rotation_create(ctx.h, f.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), f.size, int(self.interleaved),
                                    ctypes.byref(h)))
        self.h = h

    def __del__(self):
        h = getattr(self, "h", None)
        if h:
            _rotation_destroy(h)
            self.h = None


class Linear:
    """Weights of an 8-bit product with scales for each token and channel
    (palq_linear_create): w int8 [n_out, n_in], w_scale fp32 [n_out], bias
    fp32 [n_out] or None; copied."""

    def __init__(self, ctx: Context, w, w_scale, bias=None, max_rows=0):
        if w.dtype != torch.int8:
            raise PalqError(ERR_ARG, "w must be int8")
        self.ctx, (self.n_out, self.n_in) = ctx, w.shape
        _need(w_scale, torch.float32, self.n_out, "w_scale")
        if bias is not None:
            _need(bias, torch.float32, self.n_out, "bias")
            _on(ctx, bias)
        _on(ctx, w, w_scale)
        _, w_ld = _rows2(w)
        h = c_p()
        ctx._check(_linear_create(ctx.h, w.data_ptr(), w_ld, w_scale.data_ptr(), _ptr(bias), self.n_out, self.n_in, max_rows,
                                  ctypes.byref(h)))
        self.h = h

    def kernels(self, rows) -> str:
        return _linear_kernels(self.h, rows).decode()

    def run(self, x, y, x_scale=None):
        """y [rows, n_out] from x [rows, n_in]: floating values, or int8 codes with x_scale fp32 [rows]."""
        (rows, n_in), (y_rows, n_out) = x.shape, y.shape
        if n_in != self.n_in or y_rows != rows or n_out != self.n_out:
            raise PalqError(ERR_ARG, "x or y does not have the layer's shape")
        xt, x_ld = _rows2(x)
        yt, y_ld = _rows2(y)
        d = self.ctx.device
        if d >= 0 and (x.get_device() != d or y.get_device() != d):
            _on(self.ctx, x, y)
        if x_scale is not None:
            _need(x_scale, torch.float32, rows, "x_scale")
            _on(self.ctx, x_scale)
            x_scale = x_scale.data_ptr()
        st = _linear_run(self.ctx.h, self.h, x.data_ptr(), xt, x_ld, x_scale, rows, y.data_ptr(), yt, y_ld)
        if st:
            self.ctx._check(st)

    def __del__(self):
        h = getattr(self, "h", None)
        if h:
            _linear_destroy(h)
            self.h = None


class Cache:
    """A paged 8-bit key/value cache (palq_cache) over tensors of the caller:
    k int8 [pages, heads, page_tokens, head_dim], v int8 [pages, heads,
    head_dim, page_tokens], k_scale and v_scale fp32 [pages, heads]."""

    def __init__(self, k, v, k_scale, v_scale):
        pages, heads, page, dim = k.shape
        if tuple(v.shape) != (pages, heads, dim, page) or k.dtype != torch.int8 or v.dtype != torch.int8:
            raise PalqError(ERR_ARG, "k and v must be int8 [pages, heads, page, dim] and [pages, heads, dim, page]")
        if not k.is_contiguous() or not v.is_contiguous():
            raise PalqError(ERR_ARG, "k and v must be contiguous")
        _need(k_scale, torch.float32, pages * heads, "k_scale")
        _need(v_scale, torch.float32, pages * heads, "v_scale")
        self.device = _together(k, v, k_scale, v_scale)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page, self.dim = pages, heads, page, dim
        self.desc = CacheDesc(pages, page, heads, dim, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self.ref = ctypes.byref(self.desc)

    @staticmethod
    def empty(pages, heads, page, dim, device="cuda"):
        """A cache on memory of its own; every code 0."""
        return Cache(torch.zeros(pages, heads, page, dim, dtype=torch.int8, device=device),
                     torch.zeros(pages, heads, dim, page, dtype=torch.int8, device=device),
                     torch.ones(pages, heads, device=device), torch.ones(pages, heads, device=device))


class Batch:
    """A batch of requests (palq_batch): table int32 [requests, max_pages],
    lens int32 [requests], starts int32 [requests + 1] on the device, and the
    host's bounds for rows and tokens of one request."""

    def __init__(self, table, lens, starts, max_new, max_len):
        requests, max_pages = table.shape
        if table.dtype != torch.int32 or not table.is_contiguous():
            raise PalqError(ERR_ARG, "table must be contiguous int32")
        _need(lens, torch.int32, requests, "lens")
        _need(starts, torch.int32, requests + 1, "starts")
        if max_new < 0 or max_len < 0:
            raise PalqError(ERR_ARG, "max_new and max_len must be 0 or more")
        max_new, max_len = min(max_new, _INT_MAX), min(max_len, _INT_MAX)
        self.device = _together(table, lens, starts)
        self.table, self.lens, self.starts, self.tokens = table, lens, starts, 0
        self.desc = BatchDesc(requests, max_pages, table.data_ptr(), lens.data_ptr(), starts.data_ptr(), 0, max_new, max_len)
        self.ref = ctypes.byref(self.desc)


def _need(t, dtype, n, what):
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise PalqError(ERR_ARG, f"{what} must be {n} contiguous values of {dtype}")


def _on(ctx, *tensors):
    """A kernel reads whatever address it is given: tensors have to be on the context's device (no matter where for a
    validate-only one)."""
    d = ctx.device
    if d >= 0:
        for t in tensors:
            if t.get_device() != d:
                raise PalqError(ERR_ARG, f"a tensor is on {t.device}, the context on cuda:{d}")


def _together(*tensors):
    """The one device of some tensors (-1: the host)."""
    d = tensors[0].get_device()
    if any(t.get_device() != d for t in tensors):
        raise PalqError(ERR_ARG, "the tensors are on different devices")
    return d


def _tree(ctx, t, tokens):
    """Masks of a tree of drafted tokens, int64 [tokens, words], as the library takes them."""
    shape = t.shape
    if t.dtype != torch.int64 or len(shape) != 2 or shape[0] != tokens or not t.is_contiguous():
        raise PalqError(ERR_ARG, "tree must be contiguous int64 [tokens, words]")
    if ctx.device >= 0 and t.get_device() != ctx.device:
        _on(ctx, t)
    return ctypes.byref(TreeDesc(t.data_ptr(), shape[1]))


def _rows2(t):
    """Type and row stride of a [rows, cols] tensor with consecutive columns."""
    ld, one = t.stride()
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise PalqError(ERR_ARG, f"no element type for {t.dtype}")
    rows, cols = t.shape
    if one != 1 and cols > 1:
        raise PalqError(ERR_ARG, "a row's elements must be consecutive")
    return kind, (ld if rows > 1 else max(ld, cols))


def _pair3(ctx, a, b, batch, cache, query=False):
    """Type, and row and head strides of both, of two [tokens, heads, head_dim]
    tensors of a batch (query: of any multiple of the cache's heads)."""
    tokens, heads, dim = a.shape
    ar, ah, a1 = a.stride()
    br, bh, b1 = b.stride()
    kind = _TYPES.get(a.dtype)
    if a.dtype != b.dtype or b.shape != a.shape or kind is None:
        raise PalqError(ERR_ARG, "the tensors differ in type or shape, or have no element type of the library")
    if a1 != 1 or b1 != 1 or dim != cache.dim or (heads % cache.heads if query else heads != cache.heads):
        raise PalqError(ERR_ARG, "tensors must be [tokens, heads, head_dim] of the cache, a head's channels consecutive")
    d = ctx.device
    if d >= 0 and not (a.get_device() == d and b.get_device() == d and cache.device == d and batch.device == d):
        raise PalqError(ERR_ARG, f"tensors, cache or batch are not on the context's device, cuda:{d}")
    if batch.tokens != tokens:
        batch.tokens = batch.desc.tokens = tokens
    return kind, ar, ah, br, bh


class ConvPlan:
    """A planned layer (palq_conv_plan_create): the filter, requant arrays
    and shortcut scale are consumed at creation; run() takes tensors of the
    planned shapes."""

    def __init__(self, ctx: Context, x: Tensor, w: Filter, stride, pad, mult, shift, bias, out: Tensor,
                 shuffle=0, identity: Tensor = None, res_mult=None, proj_in: Tensor = None,
                 proj_w: Filter = None, proj_stride=1):
        self.ctx = ctx
        rq = Requant(_ptr(mult), _ptr(shift), _ptr(bias), out.act.bits)
        res = None
        if identity is not None or proj_in is not None:
            res = Residual()
            if identity is not None:
                res.identity = ctypes.pointer(identity.act)
                res.res_mult = _ptr(res_mult)
            if proj_in is not None:
                res.proj_in = ctypes.pointer(proj_in.act)
                res.proj_w = ctypes.pointer(proj_w)
                res.proj_stride = proj_stride
        h = c_p()
        ctx._check(_conv_plan_create(ctx.h, ctypes.byref(x.act), ctypes.byref(w), stride, pad, ctypes.byref(rq),
                                     ctypes.byref(res) if res is not None else None, shuffle,
                                     ctypes.byref(out.act), ctypes.byref(h)))
        self.h = h

    @property
    def kernels(self) -> str:
        return _conv_plan_kernels(self.h).decode()

    def run(self, x: Tensor, out: Tensor, res_in: Tensor = None, acc_dump=None):
        self.ctx._check(_conv_run(self.ctx.h, self.h, x.act.data, res_in.act.data if res_in is not None else None,
                                  out.act.data, _ptr(acc_dump)))

    def __del__(self):
        h = getattr(self, "h", None)
        if h:
            _conv_plan_destroy(h)
            self.h = None


class Net:
    """A network built from the layer-spec list of paper_2208_01944_amd.inputs."""

    def __init__(self, ctx: Context, spec, flags=0):
        self.ctx = ctx
        self.spec = spec
        self._keep = []  # device copies alive until palq_net_create has copied them
        x = spec["x"]
        n, h, w, c = x.shape
        self.input_act = make_act(n, h, w, 1, c, 8, True)
        layers = (Layer * len(spec["layers"]))()
        i32 = lambda a: self._dev(np.asarray(a, np.int32))
        for i, L in enumerate(spec["layers"]):
            d = layers[i]
            d.src, d.dst = L["src"], L["dst"]
            d.res_src = -1
            d.proj_src = -1
            if L["op"] == "conv":
                d.op = OP_CONV
                wb = int(L["w_bits"])
                wt, d.w = ctx.pack_filter(L["w"], wb)
                self._keep.append(wt)
                d.stride, d.pad = L["stride"], L["pad"]
                d.mult, d.shift = i32(L["mult"]), i32(L["shift"])
                d.bias = i32(L["bias"]) if L.get("bias") is not None else None
                d.out_bits = L["out_bits"]
                d.shuffle_steps = L.get("shuffle", 0)
                if L.get("res", -1) >= 0:
                    d.res_src = L["res"]
                    d.res_mult = i32(L["res_mult"])
                if L.get("proj_src", -1) >= 0:
                    d.proj_src = L["proj_src"]
                    pt, d.proj_w = ctx.pack_filter(L["proj_w"], wb)
                    self._keep.append(pt)
                    d.proj_stride = L["proj_stride"]
            elif L["op"] == "shuffle_module":
                d.op = OP_SHUFFLE_MODULE
                wt, d.w = ctx.pack_filter(L["w"], int(L["w_bits"]))
                self._keep.append(wt)
                d.mult, d.shift = i32(L["mult"]), i32(L["shift"])
                d.bias = i32(L["bias"]) if L.get("bias") is not None else None
                d.out_bits = L["out_bits"]
                d.res_mult = i32(L["res_mult"])
            elif L["op"] == "channel_shuffle":
                d.op = OP_CHANNEL_SHUFFLE
            elif L["op"] == "maxpool":
                d.op = OP_MAXPOOL
                d.pool_k, d.pool_stride, d.pool_pad = L["k"], L["stride"], L["pad"]
            elif L["op"] == "avgsum":
                d.op = OP_AVGSUM
            elif L["op"] == "fc":
                d.op = OP_FC
                d.fc_w = self._dev(np.asarray(L["w"], np.int8))
                d.fc_out = L["w"].shape[0]
            else:
                raise ValueError(L["op"])
        self.n_layers = len(spec["layers"])
        self.classes = spec["layers"][-1]["w"].shape[0]
        h = c_p()
        ctx._check(_net_create(ctx.h, ctypes.byref(self.input_act), layers, len(spec["layers"]),
                               flags, ctypes.byref(h)))
        self.h = h
        self._keep = []

    def _dev(self, arr):
        t = self.ctx.upload(arr)
        self._keep.append(t)
        return t.data_ptr()

    def __del__(self):
        h = getattr(self, "h", None)
        if h:
            _net_destroy(h)
            self.h = None

    @property
    def ops(self) -> int:
        return int(_net_ops(self.h))

    @staticmethod
    def _require(t, nbytes, what):
        """The C calls take plain pointers: refuse a torch tensor smaller than
        the network's batch needs before handing it over."""
        if hasattr(t, "numel") and t.numel() * t.element_size() < nbytes:
            raise PalqError(ERR_ARG, f"{what} holds fewer bytes than the network's batch needs")

    def forward(self, x_packed, logits):
        a = self.input_act
        self._require(x_packed, act_bytes(a), "input")
        self._require(logits, 4 * a.n * self.classes, "logits")
        self.ctx._check(_forward(self.ctx.h, self.h, _ptr(x_packed), _ptr(logits)))

    def forward_image(self, x_f32, l, u, logits):
        """palq_forward_image: quantise an fp32 [n][h][w][3] image (Eq. 2,
        fixed l, u) and run the network on it."""
        a = self.input_act
        self._require(x_f32, 4 * a.n * a.h * a.w * a.ch_per_group, "input")
        self._require(logits, 4 * a.n * self.classes, "logits")
        self.ctx._check(_forward_image(self.ctx.h, self.h, _ptr(x_f32), float(l), float(u), _ptr(logits)))

    def tensor(self, tid) -> Tensor:
        a = Act()
        st = _net_tensor(self.h, tid, ctypes.byref(a))
        if st != OK:
            raise PalqError(st, f"no tensor {tid}")
        return Tensor(None, a)

    def layer_kernels(self, image=False):
        """The kernels each layer launches in palq_forward (or, image=True,
        palq_forward_image), as the library's selection picked them."""
        out = []
        for i in range(self.n_layers):
            r = _net_layer_kernels(self.h, i, int(bool(image)))
            if r is None:
                raise PalqError(ERR_ARG, f"palq_net_layer_kernels({i})")
            out.append(r.decode())
        return out

    def input_kernel(self):
        """palq_forward_image's own quantiser pass ("" when the stem's
        bordered input takes the codes directly)."""
        return _net_layer_kernels(self.h, -1, 1).decode()

    def layer_times(self):
        ms = (c_f * self.n_layers)()
        fw = c_i32()
        self.ctx._check(_net_layer_times(self.h, ms, ctypes.byref(fw)))
        return np.array(ms[:], dtype=np.float64), fw.value

    def reset_times(self):
        self.ctx._check(_net_reset_times(self.h))
