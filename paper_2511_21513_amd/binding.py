"""Thin ctypes binding of the C ABI in ``include/intattn.h``.

Argument marshalling only: torch supplies device memory and the stream, every step of the
attention path runs inside ``libintattn.so``.  There is no fallback: if the library has not
been built (``python -m paper_2511_21513_amd.build`` or ``__graft_entry__.build()``), loading
raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libintattn.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_HIP, ERR_NOMEM = 0, -1, -2, -3, -4

SYMBOLS = (
    "intattn_create",
    "intattn_forward",
    "intattn_forward_noalloc",
    "intattn_reserve",
    "intattn_forward_stage",
    "intattn_forward_dynamic",
    "intattn_dynamic_status",
    "intattn_forward_quantonly",
    "intattn_quantize",
    "intattn_quantize_batch",
    "intattn_index_softmax",
    "intattn_rope",
    "intattn_cache_append",
    "intattn_cache_forward",
    "intattn_cache_evict",
    "intattn_cache_reserve",
    "intattn_derive_params",
    "intattn_derive_index_map",
    "intattn_kernel_choice",
    "intattn_get_lut",
    "intattn_last_error",
    "intattn_destroy",
)


class IntAttnError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"intattn error {code}: {text}")
        self.code = code


class Config(ctypes.Structure):
    _fields_ = [
        ("device", ctypes.c_int32),
        ("lut_bits", ctypes.c_int32),
        ("clip", ctypes.c_double),
        ("variant", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


class Args(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
        ("L", ctypes.c_int32), ("d", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
        ("scale_mode", ctypes.c_int32), ("Lkv", ctypes.c_int32),
        ("scale_q", ctypes.c_void_p), ("scale_k", ctypes.c_void_p),
        ("scale_v", ctypes.c_void_p), ("scale_out", ctypes.c_void_p),
        ("dbg_row_max", ctypes.c_void_p), ("dbg_row_sum", ctypes.c_void_p), ("dbg_acc", ctypes.c_void_p),
        ("q_block", ctypes.c_int32), ("k_block", ctypes.c_int32),
    ]


_ARGS = struct.Struct("@6i4P12q2i7P2i")  # the same, with the padding of the platform
assert _ARGS.size == ctypes.sizeof(Args)


class SoftmaxArgs(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("c_int", ctypes.c_int32),
        ("logits", ctypes.c_void_p), ("prob", ctypes.c_void_p),
        ("logits_stride", ctypes.c_int64), ("prob_stride", ctypes.c_int64),
        ("causal", ctypes.c_int32), ("rows_per_matrix", ctypes.c_int32),
    ]


class QuantArgs(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("scale_mode", ctypes.c_int32),
        ("src", ctypes.c_void_p), ("dst", ctypes.c_void_p),
        ("src_stride", ctypes.c_int64 * 3), ("dst_stride", ctypes.c_int64 * 3),
        ("scales", ctypes.c_void_p),
        ("q_block", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class Cache(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
        ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("scale_mode", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("lens", ctypes.c_void_p),
        ("scale_k", ctypes.c_void_p), ("scale_v", ctypes.c_void_p),
    ]


class Rotary(ctypes.Structure):
    _fields_ = [
        ("rot", ctypes.c_int32), ("pairing", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("inverse", ctypes.c_int32),
        ("pos", ctypes.c_void_p), ("pos_stride", ctypes.c_int64 * 3), ("freq", ctypes.c_void_p), ("axis", ctypes.c_uint8 * 128),
    ]


class RopeArgs(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("H", ctypes.c_int32 * 2),
        ("src", ctypes.c_void_p * 2), ("dst", ctypes.c_void_p * 2),
        ("src_stride", (ctypes.c_int64 * 3) * 2), ("dst_stride", (ctypes.c_int64 * 3) * 2), ("rotary", Rotary),
    ]


class AppendArgs(ctypes.Structure):
    _fields_ = [
        ("L", ctypes.c_int32), ("Hq", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("n_new", ctypes.c_void_p), ("q_out", ctypes.c_void_p), ("q_out_stride", ctypes.c_int64 * 3), ("q_scale", ctypes.c_void_p),
        ("rotary", Rotary), ("weight", ctypes.c_void_p), ("order", ctypes.c_void_p), ("first", ctypes.c_void_p),
        ("weight_stride", ctypes.c_int64 * 2), ("order_stride", ctypes.c_int64 * 2),
    ]


class CacheForwardArgs(ctypes.Structure):
    _fields_ = [
        ("Hq", ctypes.c_int32), ("L", ctypes.c_int32), ("max_len", ctypes.c_int32), ("out_type", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64 * 3), ("scale_q", ctypes.c_void_p), ("n_new", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64 * 3), ("scale_out", ctypes.c_void_p),
        ("weight", ctypes.c_void_p), ("weight_out", ctypes.c_void_p),
        ("weight_stride", ctypes.c_int64 * 2), ("weight_out_stride", ctypes.c_int64 * 2),
        ("decay", ctypes.c_float), ("scale_out_mode", ctypes.c_int32),
    ]


class EvictArgs(ctypes.Structure):
    _fields_ = [
        ("keep", ctypes.c_int32), ("sink", ctypes.c_int32), ("recent", ctypes.c_int32), ("max_len", ctypes.c_int32),
        ("weight", ctypes.c_void_p), ("weight_out", ctypes.c_void_p), ("order", ctypes.c_void_p), ("order_out", ctypes.c_void_p),
        ("weight_stride", ctypes.c_int64 * 2), ("weight_out_stride", ctypes.c_int64 * 2),
        ("order_stride", ctypes.c_int64 * 2), ("order_out_stride", ctypes.c_int64 * 2),
        ("total", ctypes.c_void_p), ("lens_out", ctypes.c_void_p),
    ]


# the argument structs as one pack each, with the padding of the platform (an assignment for each field took most of a call's time)
_ROTARY = "4iP3qP128s"
_ROPE = struct.Struct("@4i2i2P2P6q6q" + _ROTARY)
_APPEND = struct.Struct("@4i3P9qPP3qP" + _ROTARY + "3P4q")
_CACHE_FORWARD = struct.Struct("@4iP3qPPP3qPPP4qfi")
_EVICT = struct.Struct("@4i4P8q2P")
for _s, _c in ((_ROPE, RopeArgs), (_APPEND, AppendArgs), (_CACHE_FORWARD, CacheForwardArgs), (_EVICT, EvictArgs)):
    assert _s.size == ctypes.sizeof(_c)
_NO_ROTATION = (0, 0, 0, 0, 0, 0, 0, 0, 0, b"")

_lib = None
_F32 = np.dtype(np.float32)


def load() -> ctypes.CDLL:
    """Loads libintattn.so (raises if it is not built) and declares the prototypes."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2511_21513_amd.build` "
                "(there is no fallback path)"
            )
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        lib.intattn_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Config)]
        lib.intattn_create.restype = i32
        lib.intattn_forward.argtypes = [vp, ctypes.POINTER(Args), vp]
        lib.intattn_forward.restype = i32
        lib.intattn_forward_noalloc.argtypes = [vp, ctypes.POINTER(Args), vp]
        lib.intattn_forward_noalloc.restype = i32
        lib.intattn_reserve.argtypes = [vp, ctypes.POINTER(Args), i32]
        lib.intattn_reserve.restype = i32
        lib.intattn_forward_stage.argtypes = [vp, ctypes.POINTER(Args), vp, i32]
        lib.intattn_forward_stage.restype = i32
        lib.intattn_forward_dynamic.argtypes = [vp, ctypes.POINTER(Args), vp]
        lib.intattn_forward_dynamic.restype = ctypes.c_int
        lib.intattn_dynamic_status.argtypes = [vp, ctypes.POINTER(i32)]
        lib.intattn_dynamic_status.restype = ctypes.c_int
        lib.intattn_index_softmax.argtypes = [vp, ctypes.POINTER(SoftmaxArgs), vp]
        lib.intattn_index_softmax.restype = ctypes.c_int
        cache = ctypes.POINTER(Cache)  # (the other structs come packed, as bytes)
        lib.intattn_rope.argtypes = [vp, vp, vp]
        lib.intattn_cache_append.argtypes = [vp, cache, vp, vp]
        lib.intattn_cache_forward.argtypes = [vp, cache, vp, vp]
        lib.intattn_cache_evict.argtypes = [vp, cache, vp, vp]
        lib.intattn_cache_reserve.argtypes = [vp, cache, i32, i32, i32]
        for f in (lib.intattn_rope, lib.intattn_cache_append, lib.intattn_cache_forward, lib.intattn_cache_evict, lib.intattn_cache_reserve):
            f.restype = i32
        lib.intattn_quantize.argtypes = [vp, ctypes.POINTER(QuantArgs), vp]
        lib.intattn_quantize.restype = i32
        lib.intattn_quantize_batch.argtypes = [vp, ctypes.POINTER(QuantArgs), i32, vp]
        lib.intattn_quantize_batch.restype = i32
        lib.intattn_forward_quantonly.argtypes = [vp, ctypes.POINTER(Args), vp]
        lib.intattn_forward_quantonly.restype = i32
        lib.intattn_derive_params.argtypes = [
            vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float, i32,
            ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(i32), ctypes.POINTER(i32),
        ]
        lib.intattn_derive_params.restype = i32
        lib.intattn_derive_index_map.argtypes = [
            vp, ctypes.c_int64, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_uint32),
            ctypes.POINTER(ctypes.c_uint32), ctypes.POINTER(i32),
        ]
        lib.intattn_derive_index_map.restype = i32
        lib.intattn_kernel_choice.argtypes = [vp, ctypes.POINTER(Args), i32, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
        lib.intattn_kernel_choice.restype = i32
        lib.intattn_get_lut.argtypes = [vp, vp, i32]
        lib.intattn_get_lut.restype = i32
        lib.intattn_last_error.argtypes = [vp]
        lib.intattn_last_error.restype = ctypes.c_char_p
        lib.intattn_destroy.argtypes = [vp]
        lib.intattn_destroy.restype = None
        _lib = lib
    return _lib


def _host_f32(x):
    if x is None or (type(x) is np.ndarray and x.dtype == _F32 and x.ndim and x.flags.c_contiguous):
        return x
    return np.ascontiguousarray(np.atleast_1d(np.asarray(x, dtype=np.float32)))


def _address(x):
    """Address of a host array (``x.ctypes.data`` at half its time, for arrays that can be written to)."""
    try:
        return ctypes.addressof(ctypes.c_char.from_buffer(x))
    except (TypeError, ValueError):
        return x.ctypes.data


def _ptr(t):
    return t.data_ptr() if t is not None else 0


_types = {}


def _float_types():
    if not _types:
        import torch

        _types.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
    return _types


def _check(t, what, dtype, shape, device, contiguous=False):
    """A tensor (or None) that a struct will point at: its type, shape and device index, which pointers do not carry."""
    if t is not None and (t.dtype is not dtype or t.shape != shape or t.get_device() != device or (contiguous and not t.is_contiguous())):
        raise ValueError(f"{what} must be a {'contiguous ' if contiguous else ''}{dtype} tensor of shape {tuple(shape)} on cuda:{device}, "
                         f"not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows(t, what, dtype, shape, device):
    """The same for [B, H, L, d] tensors whose last axis has to be contiguous: their strides."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _check(t, what, dtype, shape, device)
    st = t.stride()
    if st[3] != 1:
        raise ValueError(f"{what}: the head dimension must be contiguous")
    return st


def _like(torch, t, dtype):
    """A new tensor in the memory order of a [B, H, L, d] tensor, where its rows can be written in pieces of 16 bytes, and its strides."""
    out = torch.empty_like(t, dtype=dtype)
    s0, s1, s2, s3 = out.stride()
    if s3 == 1 and not (s0 | s1 | s2) & 15:
        return out, s0, s1, s2
    out = torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)  # (a broadcast axis of t may end up innermost)
    return out, *out.stride()[:3]


def _slots(t, what, dtype, B, Hkv, slots, device):
    """[B, Hkv, slots] planes (or None): the last axis is contiguous and holds every slot the call may touch."""
    if t is None:
        return 0, 0
    n, st = t.shape, t.stride()
    if len(n) != 3 or n[2] < slots or st[2] != 1:
        raise ValueError(f"{what} must be [B, Hkv, slots] with at least {slots} slots, contiguous")
    if t.dtype is not dtype or n[0] != B or n[1] != Hkv or t.get_device() != device:
        _check(t, what, dtype, (B, Hkv, n[2]), device)
    return st[0], st[1]


def _rotation(torch, B, L, device, pos, freq, axis, pairing, inverse):
    """The fields of intattn_rotary."""
    if pos.dim() == 2:
        pos = pos[None]
    axes, n = pos.shape[0], freq.shape[0]
    if pos.dtype is not torch.int32 or pos.shape != (axes, B, L) or pos.get_device() != device:
        _check(pos, "pos", torch.int32, (axes, B, L), device)
    if freq.dtype is not torch.float64 or freq.dim() != 1 or freq.get_device() != device or not freq.is_contiguous():
        _check(freq, "freq", torch.float64, (n,), device, True)
    if n > 128:
        raise ValueError("at most 128 rotated pairs")
    if pairing not in ("adjacent", "halves"):
        raise ValueError("pairing is 'adjacent' or 'halves'")
    if axis is not None:
        axis = bytes(axis)  # (raises unless each is 0 .. 255; the library compares them with the axes)
        if len(axis) != n:
            raise ValueError("axis must name an axis for each pair")
    return (2 * n, int(pairing == "halves"), axes, int(bool(inverse)), pos.data_ptr(), *pos.stride(), freq.data_ptr(), axis or b"")


def _whole_rows(torch, g):
    """A gradient that autograd hands on, which may have any strides, as a tensor that the kernels can read."""
    s0, s1, s2, s3 = g.stride()
    if s3 == 1 and not (g.data_ptr() | (s0 | s1 | s2) * g.element_size()) & 15:
        return g
    return g.clone(memory_format=torch.contiguous_format)


_rope_function = None


def _differentiable_rope(torch):
    """The autograd function of ``IntAttn.rope``: its gradient is the rotation backwards, a rope itself."""
    global _rope_function
    if _rope_function is None:

        class Rope(torch.autograd.Function):
            @staticmethod
            def forward(ctx, ia, pos, freq, axis, pairing, inverse, stream, *xs):
                axis = None if axis is None else bytes(axis)  # (the caller may change the list)
                ctx.how = (ia, axis, pairing, inverse)
                ctx.save_for_backward(pos, freq)  # (changed in place before the backward pass, torch raises)
                ctx.set_materialize_grads(False)
                outs = tuple(ia.rope(xs, pos, freq, axis=axis, pairing=pairing, inverse=inverse, stream=stream))
                ctx.mark_non_differentiable(*(o for o, needed in zip(outs, ctx.needs_input_grad[7:]) if not needed))
                return outs

            @staticmethod
            def backward(ctx, *gs):
                ia, axis, pairing, inverse = ctx.how
                pos, freq = ctx.saved_tensors
                those = [i for i, g in enumerate(gs) if g is not None and ctx.needs_input_grad[7 + i]]
                grads = [None] * len(gs)
                if those:
                    got = ia.rope([_whole_rows(torch, gs[i]) for i in those], pos, freq, axis=axis, pairing=pairing, inverse=not inverse)
                    for i, g in zip(those, got):
                        grads[i] = g
                return (None,) * 7 + tuple(grads)

        _rope_function = Rope
    return _rope_function


class PagedCache:
    """A paged INT8 key/value cache (``intattn_cache``): the caller's tensors, checked once, and the struct that points at them.

    ``k_pages``, ``v_pages``: int8 [n_pages, Hkv, page_size, d]; ``table``: int32 [B, max_pages], the pages of each sequence (a
    number outside the pool: a page that is not there); ``lens``: int32 [B], keys of each sequence, which the caller keeps (in
    place); ``scale_k``, ``scale_v``: float32, one value or one for each KV head.  The contents may change between calls."""

    def __init__(self, k_pages, v_pages, table, lens, scale_k, scale_v):
        import torch

        if k_pages.dim() != 4 or not k_pages.is_cuda or table.dim() != 2:
            raise ValueError("k_pages must be an int8 tensor [n_pages, Hkv, page_size, d] on the GPU, table [B, max_pages]")
        dev = k_pages.get_device()
        n_pages, Hkv, page, d = k_pages.shape
        k_st, v_st = (_rows(t, what, torch.int8, (n_pages, Hkv, page, d), dev) for t, what in ((k_pages, "k_pages"), (v_pages, "v_pages")))
        B = table.shape[0]
        _check(table, "table", torch.int32, (B, table.shape[1]), dev)
        if table.shape[1] > 1 and table.stride(1) != 1:
            raise ValueError("rows of the table must be contiguous")
        _check(lens, "lens", torch.int32, (B,), dev, True)
        for t, what in ((scale_k, "scale_k"), (scale_v, "scale_v")):
            _check(t, what, torch.float32, (scale_k.numel(),), dev, True)
        if scale_k.numel() not in (1, Hkv):
            raise ValueError("scales: one value, or one for each KV head")
        self.k_pages, self.v_pages, self.table, self.lens, self.scale_k, self.scale_v = k_pages, v_pages, table, lens, scale_k, scale_v
        self.B, self.Hkv, self.page_size, self.d, self.device = B, Hkv, page, d, dev
        self.capacity = table.shape[1] * page
        c = Cache()
        c.B, c.Hkv, c.d, c.n_pages, c.page_size, c.max_pages = B, Hkv, d, n_pages, page, table.shape[1]
        c.scale_mode = int(scale_k.numel() == Hkv)
        c.k, c.v, c.table, c.lens = k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), lens.data_ptr()
        c.scale_k, c.scale_v = scale_k.data_ptr(), scale_v.data_ptr()
        c.k_stride[:], c.v_stride[:] = k_st[:3], v_st[:3]
        c.table_stride = table.stride(0)
        self.args = c
        self._ref = ctypes.byref(c)


class IntAttn:
    """One library context (``intattn_create`` .. ``intattn_destroy``)."""

    def __init__(self, device: int = 0, lut_bits: int = 5, clip: float = 6.6, variant: int = 0):
        self._lib = load()
        self._ctx = ctypes.c_void_p()
        cfg = Config(device, lut_bits, clip, variant, 0)
        rc = self._lib.intattn_create(ctypes.byref(self._ctx), ctypes.byref(cfg))
        if rc != OK:
            raise IntAttnError(rc, (self._lib.intattn_last_error(None) or b"").decode())
        self.device = device

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self._lib.intattn_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_error(self) -> str:
        return (self._lib.intattn_last_error(self._ctx) or b"").decode()

    def lut(self) -> np.ndarray:
        buf = np.zeros(64, dtype=np.uint8)
        n = self._lib.intattn_get_lut(self._ctx, buf.ctypes.data_as(ctypes.c_void_p), 64)
        if n < 0:
            raise IntAttnError(n, "intattn_get_lut")
        return buf[:n].copy()

    def derive_params(self, s_q, s_k, s_v, s_o, d):
        c, m, sh = ctypes.c_int64(0), ctypes.c_int32(0), ctypes.c_int32(0)
        rc = self._lib.intattn_derive_params(
            self._ctx, float(np.float32(s_q)), float(np.float32(s_k)), float(np.float32(s_v)),
            float(np.float32(s_o)), d, ctypes.byref(c), ctypes.byref(m), ctypes.byref(sh),
        )
        if rc != OK:
            raise IntAttnError(rc, "intattn_derive_params")
        return int(c.value), int(m.value), int(sh.value)

    def derive_index_map(self, c_int: int, mode: int = 2):
        mode, sh = ctypes.c_int32(mode), ctypes.c_int32(0)
        mul, add = ctypes.c_uint32(0), ctypes.c_uint32(0)
        rc = self._lib.intattn_derive_index_map(
            self._ctx, c_int, ctypes.byref(mode), ctypes.byref(mul), ctypes.byref(add), ctypes.byref(sh)
        )
        if rc != OK:
            raise IntAttnError(rc, "intattn_derive_index_map")
        return int(mode.value), int(mul.value), int(add.value), int(sh.value)

    def kernel_choice(self, args: Args, dynamic: bool = False):
        """intattn_kernel_choice: (kernel, split_rows, split_pv) for a call with these arguments."""
        out = [ctypes.c_int32(0) for _ in range(3)]
        rc = self._lib.intattn_kernel_choice(self._ctx, ctypes.byref(args), int(bool(dynamic)), *(ctypes.byref(x) for x in out))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())
        return tuple(int(x.value) for x in out)

    def make_args(self, q, k, v, out, s_q, s_k, s_v, s_o=None, *, causal=False, per_head=False,
                  row_max=None, row_sum=None, acc=None, device_scales=False, q_block=0, k_block=0):
        """Marshals torch int8 tensors [B,H,L,d] (last dim contiguous) into an ``Args``.  Returns
        (args, keepalive): keepalive holds the scale arrays the struct points at: host arrays, or
        with ``device_scales`` the float32 device tensors given (for ``forward_dynamic_args``).
        ``q_block`` > 0 (device scales only): scale mode 2, s_q and s_o hold one value per block of
        ``q_block`` query rows of every (batch, head), s_k and s_v one per KV head.  ``k_block`` > 0 as
        well: scale mode 3, s_k holds one value per block of ``k_block`` keys of every (batch, KV head)."""
        B, Hq, L, d = q.shape
        ks = k.shape
        Hkv = ks[1]
        if ks != v.shape or ks[0] != B or ks[3] != d or out.shape != q.shape:
            raise ValueError("q, out must be [B,Hq,L,d] and k, v [B,Hkv,Lkv,d]")
        strides = q.stride(), k.stride(), v.stride(), out.stride()
        for st in strides:
            if st[-1] != 1:
                raise ValueError("the head dimension must be contiguous")
        lkv = ks[2]
        if device_scales:
            import torch

            keep = [s_q, s_k, s_v, s_o]
            for t in keep:
                if t is not None and (t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous()):
                    raise ValueError("device scales must be contiguous float32 tensors on the GPU")
            sizes = [t.numel() if t is not None else None for t in keep]
            ptr = [t.data_ptr() for t in keep[:3]] + [s_o.data_ptr() if s_o is not None else 0]
        else:
            keep = [_host_f32(s_q), _host_f32(s_k), _host_f32(s_v), _host_f32(s_o)]
            sizes = [t.size if t is not None else None for t in keep]
            ptr = [_address(t) for t in keep[:3]] + [_address(keep[3]) if keep[3] is not None else 0]
        scale_mode = int(bool(per_head))
        if q_block:
            if not device_scales:
                raise ValueError("q_block needs device_scales")
            n_grp = B * Hq * ((L + q_block - 1) // q_block)
            scale_mode = 2
            want = [n_grp, Hkv, Hkv, n_grp]
            if k_block:
                scale_mode = 3
                want[1] = B * Hkv * ((lkv + k_block - 1) // k_block)
        elif k_block:
            raise ValueError("k_block needs q_block (use q_block = L for one query scale per head)")
        else:
            want = [Hq, Hkv, Hkv, Hq] if per_head else [1, 1, 1, 1]
        for have, need in zip(sizes, want):
            if have is not None and (have != need if (per_head or q_block) else have < 1):
                raise ValueError("scale arrays do not have the number of entries the scale mode needs")
        (q0, q1, q2), (k0, k1, k2), (v0, v1, v2), (o0, o1, o2) = (st[:3] for st in strides)
        # one pack instead of an assignment for each field
        a = Args.from_buffer_copy(_ARGS.pack(
            B, Hq, Hkv, L, d, int(bool(causal)), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
            q0, q1, q2, k0, k1, k2, v0, v1, v2, o0, o1, o2, scale_mode, lkv, *ptr,
            row_max.data_ptr() if row_max is not None else 0, row_sum.data_ptr() if row_sum is not None else 0,
            acc.data_ptr() if acc is not None else 0, 0, 0))
        if q_block:
            a.q_block, a.k_block = int(q_block), int(k_block or 0)
        return a, keep

    def forward_args(self, args: Args, stream: int = 0, quantonly: bool = False):
        fn = self._lib.intattn_forward_quantonly if quantonly else self._lib.intattn_forward
        rc = fn(self._ctx, ctypes.byref(args), ctypes.c_void_p(stream))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def forward_noalloc_args(self, args: Args, stream: int = 0):
        """intattn_forward_noalloc: the forward with its workspace in the library's static device array."""
        rc = self._lib.intattn_forward_noalloc(self._ctx, ctypes.byref(args), ctypes.c_void_p(stream))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def reserve(self, args: Args, dynamic: bool = False):
        """intattn_reserve: pre-size the context's device memory for problems up to this one."""
        rc = self._lib.intattn_reserve(self._ctx, ctypes.byref(args), int(bool(dynamic)))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def forward_dynamic_args(self, args: Args, stream: int = 0):
        """intattn_forward_dynamic: ``args`` built with ``device_scales=True``."""
        rc = self._lib.intattn_forward_dynamic(self._ctx, ctypes.byref(args), ctypes.c_void_p(stream))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def dynamic_status(self) -> int:
        st = ctypes.c_int32(0)
        rc = self._lib.intattn_dynamic_status(self._ctx, ctypes.byref(st))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())
        return int(st.value)

    def index_softmax(self, logits, c_int: int, *, causal: bool = False, rows_per_matrix: int = 0, out=None, stream=None):
        """intattn_index_softmax on a torch int32 tensor [..., cols] (rows contiguous, all leading
        axes collapsible to one row stride): uint8 probabilities of the same shape."""
        import torch

        cols = logits.shape[-1]
        flat = logits.reshape(-1, cols)  # a view, or torch raises on a copy below
        if flat.data_ptr() != logits.data_ptr() or flat.stride(-1) != 1:
            raise ValueError("logits must be viewable as [rows, cols] with contiguous rows")
        if out is None:
            out = torch.empty(logits.shape, dtype=torch.uint8, device=logits.device)
        oflat = out.reshape(-1, cols)
        if oflat.data_ptr() != out.data_ptr() or oflat.stride(-1) != 1 or oflat.shape[0] != flat.shape[0]:
            raise ValueError("out must be viewable as [rows, cols] with contiguous rows")
        a = SoftmaxArgs()
        a.rows, a.cols, a.c_int = flat.shape[0], cols, int(c_int)
        a.logits, a.prob = flat.data_ptr(), oflat.data_ptr()
        a.logits_stride = (flat.stride(0) if flat.shape[0] > 1 else cols) * 4
        a.prob_stride = oflat.stride(0) if oflat.shape[0] > 1 else cols
        a.causal, a.rows_per_matrix = int(bool(causal)), int(rows_per_matrix)
        if stream is None:
            stream = torch.cuda.current_stream(logits.device).cuda_stream
        rc = self._lib.intattn_index_softmax(self._ctx, ctypes.byref(a), ctypes.c_void_p(stream))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())
        return out

    def quantize(self, x, per_head: bool = False, out=None, scales=None, stream=None, q_block: int = 0):
        """intattn_quantize on a [B, H, L, d] device tensor (torch float32 / float16 / bfloat16,
        last dimension contiguous): returns (int8 tensor, float32 device tensor of 1 or H scales;
        with ``q_block`` > 0 one scale per block of ``q_block`` rows, [B, H, ceil(L / q_block)]).
        Argument marshalling only."""
        import torch

        dtypes = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
        if x.dim() != 4 or x.dtype not in dtypes or x.stride(3) != 1:
            raise ValueError("expected a [B, H, L, d] float32/float16/bfloat16 tensor with contiguous last dimension")
        B, H, L, d = x.shape
        if out is None:
            out = torch.empty((B, H, L, d), dtype=torch.int8, device=x.device)
        if scales is None:
            shape = (B, H, (L + q_block - 1) // q_block) if q_block else (H if per_head else 1,)
            scales = torch.empty(shape, dtype=torch.float32, device=x.device)
        a = QuantArgs()
        a.B, a.H, a.L, a.d = B, H, L, d
        a.dtype, a.scale_mode = dtypes[x.dtype], 2 if q_block else int(per_head)
        a.q_block = int(q_block)
        a.src, a.dst, a.scales = x.data_ptr(), out.data_ptr(), scales.data_ptr()
        es = x.element_size()
        for i in range(3):
            a.src_stride[i] = x.stride(i) * es
            a.dst_stride[i] = out.stride(i)
        st = torch.cuda.current_stream(x.device).cuda_stream if stream is None else stream
        rc = self._lib.intattn_quantize(self._ctx, ctypes.byref(a), ctypes.c_void_p(st))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())
        return out, scales

    def quant_args(self, x, out, scales, per_head: bool = False, q_block: int = 0) -> "QuantArgs":
        """Marshals one tensor of a quantizer call (see ``quantize``)."""
        import torch

        dtypes = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
        if x.dim() != 4 or x.dtype not in dtypes or x.stride(3) != 1:
            raise ValueError("expected a [B, H, L, d] float32/float16/bfloat16 tensor with contiguous last dimension")
        a = QuantArgs()
        a.B, a.H, a.L, a.d = x.shape
        a.dtype, a.scale_mode = dtypes[x.dtype], 2 if q_block else int(per_head)
        a.q_block = int(q_block)
        a.src, a.dst, a.scales = x.data_ptr(), out.data_ptr(), scales.data_ptr()
        es = x.element_size()
        for i in range(3):
            a.src_stride[i] = x.stride(i) * es
            a.dst_stride[i] = out.stride(i)
        return a

    def quantize_batch(self, xs, per_head=False, outs=None, scales=None, stream=None):
        """intattn_quantize_batch: up to four [B, H, L, d] device tensors in one pair of launches.
        ``per_head``: one flag, or one per tensor.  Returns (list of int8 tensors, list of scale tensors)."""
        import torch

        n = len(xs)
        flags = list(per_head) if isinstance(per_head, (list, tuple)) else [per_head] * n
        if outs is None:
            outs = [torch.empty(x.shape, dtype=torch.int8, device=x.device) for x in xs]
        if scales is None:
            scales = [torch.empty(x.shape[1] if f else 1, dtype=torch.float32, device=x.device) for x, f in zip(xs, flags)]
        arr = (QuantArgs * n)(*[self.quant_args(x, o, s, f) for x, o, s, f in zip(xs, outs, scales, flags)])
        st = torch.cuda.current_stream(xs[0].device).cuda_stream if stream is None else stream
        rc = self._lib.intattn_quantize_batch(self._ctx, arr, n, ctypes.c_void_p(st))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())
        return outs, scales

    def _stream(self, device, stream):
        import torch

        if device != self.device:
            raise ValueError(f"tensors on device {device}, context on device {self.device}")
        return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream

    def _done(self, rc):
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def rope(self, x, pos, freq, *, axis=None, pairing="adjacent", inverse=False, out=None, stream=None):
        """intattn_rope on a [B, H, L, d] tensor, or on two with the same B, L, d (Q and K): new tensors, or ``out``, which may be
        ``x``.  ``pos``: int32 [axes, B, L] (or [B, L]); ``freq``: float64 [rot / 2], radians per position of each pair, on the
        device; ``axis``: a list of each pair's axis (None: all the first).  ``inverse``: the gradient's rotation, which autograd
        takes by itself where x requires a gradient (then there is no ``out``, and ``freq`` has no gradient of its own)."""
        import torch

        one = torch.is_tensor(x)
        xs = (x,) if one else x
        n = len(xs)
        if not 1 <= n <= 2:
            raise ValueError("one tensor or two, and as many outputs")
        a, b = xs[0], xs[-1]
        if torch.is_grad_enabled():
            if freq.requires_grad:
                raise ValueError("freq has no gradient: detach it")
            if out is not None and (a.requires_grad or b.requires_grad or any(t.requires_grad for t in ([out] if torch.is_tensor(out) else out))):
                raise ValueError("out does not go with tensors that require a gradient")
            if a.requires_grad or b.requires_grad:
                outs = _differentiable_rope(torch).apply(self, pos, freq, axis, pairing, inverse, stream, *xs)
                return outs[0] if one else list(outs)
        B, H, L, d = shape = a.shape
        dtype, dev, es = a.dtype, a.get_device(), a.element_size()
        code = _float_types().get(dtype)
        if code is None:
            raise ValueError("expected float32/float16/bfloat16 tensors")
        s0, s1, s2, _ = _rows(a, "x", dtype, shape, dev)
        if n == 2:
            H2 = b.shape[1]
            t0, t1, t2, _ = _rows(b, "x", dtype, (B, H2, L, d), dev)
        else:
            H2, t0, t1, t2 = 0, s0, s1, s2
        given = out is not None
        if not given:
            o, o0, o1, o2 = p, p0, p1, p2 = _like(torch, a, dtype)
            if n == 2:
                p, p0, p1, p2 = _like(torch, b, dtype)
            out = o if one else [o, p][:n]
        else:
            outs = [out] if torch.is_tensor(out) else list(out)
            if len(outs) != n:
                raise ValueError("one tensor or two, and as many outputs")
            o, p = outs[0], outs[-1]
            o0, o1, o2, _ = _rows(o, "out", dtype, shape, dev)
            p0, p1, p2, _ = _rows(p, "out", dtype, b.shape, dev)
            out = o if one else outs
        args = _ROPE.pack(B, L, d, code, H, H2, a.data_ptr(), b.data_ptr(), o.data_ptr(), p.data_ptr(),
                          s0 * es, s1 * es, s2 * es, t0 * es, t1 * es, t2 * es, o0 * es, o1 * es, o2 * es, p0 * es, p1 * es, p2 * es,
                          *_rotation(torch, B, L, dev, pos, freq, axis, pairing, inverse))
        self._done(self._lib.intattn_rope(self._ctx, args, self._stream(dev, stream)))
        if given:
            torch.autograd.graph.increment_version(outs)  # (a graph that has kept one of them raises in its backward pass)
        return out

    def cache_append(self, cache: PagedCache, k, v, q=None, *, n_new=None, pos=None, freq=None, axis=None, pairing="adjacent",
                     weight=None, order=None, first=None, q_out=None, q_scale=None, stream=None):
        """intattn_cache_append: K and V [B, Hkv, L, d] of new tokens into the last slots of ``cache.lens`` (which already count
        them), rotated if ``pos`` and ``freq`` are given (see ``rope``).  With Q [B, Hq, L, d]: returns its INT8 tensor and the scales
        [B, Hq, L]."""
        import torch

        dev, B, L, d, dtype = cache.device, cache.B, k.shape[2], cache.d, k.dtype
        code = _float_types().get(dtype)
        if code is None:
            raise ValueError("expected float32/float16/bfloat16 tensors")
        es, shape = k.element_size(), (B, cache.Hkv, L, d)
        k0, k1, k2, _ = _rows(k, "k", dtype, shape, dev)
        v0, v1, v2, _ = _rows(v, "v", dtype, shape, dev)
        _check(n_new, "n_new", torch.int32, (B,), dev, True)
        Hq = q0 = q1 = q2 = o0 = o1 = o2 = 0
        if q is not None:
            Hq = q.shape[1]
            q0, q1, q2, _ = _rows(q, "q", dtype, (B, Hq, L, d), dev)
            if q_out is None:
                q_out, o0, o1, o2 = _like(torch, q, torch.int8)
            else:
                o0, o1, o2, _ = _rows(q_out, "q_out", torch.int8, (B, Hq, L, d), dev)
            if q_scale is None:
                q_scale = q.new_empty((B, Hq, L), dtype=torch.float32)
            else:
                _check(q_scale, "q_scale", torch.float32, (B, Hq, L), dev, True)
        planes = (0, 0, 0, 0, 0, 0, 0)
        if weight is not None or order is not None:
            _check(first, "first", torch.int32, (B,), dev, True)
            planes = (_ptr(weight), _ptr(order), _ptr(first), *_slots(weight, "weight", torch.float32, B, cache.Hkv, cache.capacity, dev),
                      *_slots(order, "order", torch.int32, B, cache.Hkv, cache.capacity, dev))
        args = _APPEND.pack(L, Hq, code, 0, _ptr(q), k.data_ptr(), v.data_ptr(), q0 * es, q1 * es, q2 * es, k0 * es, k1 * es, k2 * es,
                            v0 * es, v1 * es, v2 * es, _ptr(n_new), _ptr(q_out) if Hq else 0, o0, o1, o2, _ptr(q_scale) if Hq else 0,
                            *(_NO_ROTATION if pos is None else _rotation(torch, B, L, dev, pos, freq, axis, pairing, False)), *planes)
        self._done(self._lib.intattn_cache_append(self._ctx, cache._ref, args, self._stream(dev, stream)))
        return (q_out, q_scale) if q is not None else None

    def cache_forward(self, cache: PagedCache, q, scale_q, *, out=None, dtype=None, scale_out=None, n_new=None, max_len=0,
                      weight=None, weight_out=None, decay=1.0, stream=None):
        """intattn_cache_forward: INT8 queries [B, Hq, L, d] of the newest tokens, with a scale for each token and head, over the
        cache.  Returns ``out`` (given, or new in ``dtype`` and q's memory order; the default is torch.bfloat16, torch.int8 is the
        requantized form).  ``weight``
        [B, Hkv, slots] float32: accumulated attention weight of each key, written to ``weight_out`` (default: in place)."""
        import torch

        dev, B, Hq, L, d = cache.device, cache.B, q.shape[1], q.shape[2], cache.d
        shape = (B, Hq, L, d)
        q0, q1, q2, _ = _rows(q, "q", torch.int8, shape, dev)
        _check(scale_q, "scale_q", torch.float32, (B, Hq, L), dev, True)
        _check(n_new, "n_new", torch.int32, (B,), dev, True)
        if dtype is None:
            dtype = torch.bfloat16 if out is None else out.dtype
        code = 3 if dtype is torch.int8 else _float_types().get(dtype)
        if code is None:
            raise ValueError("out must be float32/float16/bfloat16/int8")
        if out is None:
            out, o0, o1, o2 = _like(torch, q, dtype)
        else:
            o0, o1, o2, _ = _rows(out, "out", dtype, shape, dev)
        es = out.element_size()
        per_head = int(scale_out is not None and scale_out.numel() > 1)
        _check(scale_out, "scale_out", torch.float32, (Hq if per_head else 1,), dev, True)
        planes = (0, 0, 0, 0, 0, 0)
        if weight is not None:
            slots = min(cache.capacity, max_len) if max_len else cache.capacity
            weight_out = weight if weight_out is None else weight_out
            w = _slots(weight, "weight", torch.float32, B, cache.Hkv, slots, dev)
            planes = (weight.data_ptr(), weight_out.data_ptr(), *w, *(w if weight_out is weight else _slots(weight_out, "weight_out", torch.float32, B, cache.Hkv, slots, dev)))
        elif weight_out is not None:
            raise ValueError("weight_out needs weight")
        args = _CACHE_FORWARD.pack(Hq, L, int(max_len), code, q.data_ptr(), q0, q1, q2, scale_q.data_ptr(), _ptr(n_new), out.data_ptr(),
                                   o0 * es, o1 * es, o2 * es, _ptr(scale_out), *planes, float(decay), per_head)
        self._done(self._lib.intattn_cache_forward(self._ctx, cache._ref, args, self._stream(dev, stream)))
        return out

    def cache_evict(self, cache: PagedCache, keep: int, weight, *, order=None, total=None, sink=0, recent=0, max_len=0,
                    weight_out=None, order_out=None, lens_out=None, stream=None):
        """intattn_cache_evict: sequences longer than ``keep`` keep the keys of each head that have drawn most ``weight``
        [B, Hkv, slots], among them the first ``sink`` and the last ``recent`` by ``order`` (int32 [B, Hkv, slots]; ``total`` [B]: tokens so
        far).  weight, order and lens change in place unless ``*_out`` tensors are given."""
        import torch

        dev, B, Hkv = cache.device, cache.B, cache.Hkv
        slots = min(cache.capacity, max_len) if max_len else cache.capacity
        weight_out = weight if weight_out is None else weight_out
        order_out = order if order_out is None else order_out
        lens_out = cache.lens if lens_out is None else lens_out
        _check(total, "total", torch.int32, (B,), dev, True)
        _check(lens_out, "lens_out", torch.int32, (B,), dev, True)
        w, o = _slots(weight, "weight", torch.float32, B, Hkv, slots, dev), _slots(order, "order", torch.int32, B, Hkv, slots, dev)
        planes = (*w, *(w if weight_out is weight else _slots(weight_out, "weight_out", torch.float32, B, Hkv, slots, dev)),
                  *o, *(o if order_out is order else _slots(order_out, "order_out", torch.int32, B, Hkv, slots, dev)))
        args = _EVICT.pack(int(keep), int(sink), int(recent), int(max_len), _ptr(weight), _ptr(weight_out), _ptr(order), _ptr(order_out),
                           *planes, _ptr(total), lens_out.data_ptr())
        self._done(self._lib.intattn_cache_evict(self._ctx, cache._ref, args, self._stream(dev, stream)))

    def cache_reserve(self, cache: PagedCache, rows: int = 0, keep: int = 0, max_len: int = 0):
        """intattn_cache_reserve: room for ``cache_forward`` with up to ``rows`` = Hq / Hkv * L rows a KV head and for ``cache_evict``
        to ``keep`` keys, so that they can be captured."""
        rc = self._lib.intattn_cache_reserve(self._ctx, ctypes.byref(cache.args), int(rows), int(keep), int(max_len))
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def forward_stage(self, args: Args, stage: int, stream: int = 0):
        """intattn_forward_stage: 0 = everything, 1 = sweeps A+B, 2 = sweep C."""
        rc = self._lib.intattn_forward_stage(self._ctx, ctypes.byref(args), ctypes.c_void_p(stream), stage)
        if rc != OK:
            raise IntAttnError(rc, self.last_error())

    def forward(self, q, k, v, s_q, s_k, s_v, s_o=None, *, causal=False, per_head=False, out=None,
                taps=False, stream=None, quantonly=False):
        """intattn_forward on torch tensors.  Returns ``out`` (int8 [B,Hq,L,d]); with ``taps`` a
        dict with out, row_max, row_sum, acc.  Enqueued on torch's current stream unless given."""
        import torch

        if out is None:
            out = torch.empty_like(q)
        extra = {}
        if taps:
            B, Hq, L, d = q.shape
            extra = {
                "row_max": torch.zeros((B, Hq, L), dtype=torch.int32, device=q.device),
                "row_sum": torch.zeros((B, Hq, L), dtype=torch.int32, device=q.device),
                "acc": torch.zeros((B, Hq, L, d), dtype=torch.int32, device=q.device),
            }
        args, keep = self.make_args(q, k, v, out, s_q, s_k, s_v, s_o, causal=causal, per_head=per_head, **extra)
        if stream is None:
            # the handle alone, without a Stream object around it
            stream = torch._C._cuda_getCurrentRawStream(q.device.index) if q.is_cuda else torch.cuda.current_stream(q.device).cuda_stream
        self.forward_args(args, stream, quantonly)
        del keep
        if taps:
            extra["out"] = out
            return extra
        return out
