"""Python binding of the C ABI in ``include/taps_mx.h`` (ctypes): a paged cache
held in microscaling formats of 4 or 8 bits, beside the 16-bit cache of ``attention``.

    k_cache, v_cache = (mx.new_pages(n_pages, kv_heads=8, page_size=64, head_dim=128, bits=4)
                        for _ in range(2))
    mx.taps_mx_append(k, v, k_cache, v_cache, plan, table=table, k_weight=k_weight)
    out = mx.taps_mx_attend(q, k_cache, v_cache, plan)     # plan: an attention.PagedPlan
    k, v = mx.taps_mx_read(k_cache, v_cache, slots, head_dim=128)

Argument marshalling only, as in ``attention``: every step runs in
``libtaps_attention.so``, which raises if it is missing; outputs and workspaces come from
torch's allocator, on the stream that the call runs on.  A cache has no
gradients: a backward pass through the new outputs of ``taps_mx_attend`` raises, as does
the call on queries with tangents (forward mode).
"""
from __future__ import annotations

import ctypes as C
import os
import re
from typing import List

import torch

from . import attention
from .attention import (AppendArgs, Heads, PagedPlan, _DTYPES, _check, _device, _dtype, _heads,
                        _like, _no_gradient, _on, _on_gpu, _output, _stream, _table, _vector)

HEADER = os.path.join(os.path.dirname(attention.HEADER), "taps_mx.h")

BLOCK = 32      # elements that share a scale
NAN = 255       # scale of a block that is read as NaN


class Pages(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("codes_stride", C.c_int64 * 3),
                ("scales", C.c_void_p), ("scales_stride", C.c_int64 * 3)]


class ReadArgs(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("bits", C.c_uint32), ("tokens", C.c_uint32),
                ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("page_size", C.c_uint32),
                ("n_pages", C.c_uint32), ("slot_bytes", C.c_uint32), ("slots", C.c_void_p)]


_lib = None


def load():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = attention.load()
        P = C.POINTER
        H, M = P(Heads), P(Pages)
        L.taps_mx_append.restype = C.c_int
        L.taps_mx_append.argtypes = [P(AppendArgs), C.c_uint32, C.c_void_p, C.c_void_p, H, H, M, M,
                                     C.c_void_p]
        L.taps_mx_read.restype = C.c_int
        L.taps_mx_read.argtypes = [P(ReadArgs), M, M, H, H, C.c_void_p]
        L.taps_mx_attend.restype = C.c_int
        L.taps_mx_attend.argtypes = [C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p, H, M, M,
                                     C.c_float, H, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
        _lib = L
    return _lib


def declared_symbols() -> List[str]:
    """Entry points declared in include/taps_mx.h."""
    with open(HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"^\s*taps_status\s*(taps_\w+)\s*\(", text, flags=re.M)))


class MxPages:
    """Pages of keys or of values: codes and scales, 8-bit unsigned tensors [pages, kv_heads,
    page_size, bytes] of any strides but the last.  A slot has a byte of ``scales`` for every 32
    elements of a head, and 16 (4 bits) or 32 (8 bits) of ``codes``.  They are looked at once,
    here: what they hold may change, their sizes and places may not.  Other tensors are other
    pages, and a call with tensors that have moved since (``resize_``, ``set_``) raises."""

    __slots__ = "_codes", "_scales", "_bits", "_n", "_shape", "_device", "_at", "_places"

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        for x, name in ((codes, "codes"), (scales, "scales")):
            if x.dtype is not torch.uint8:
                raise ValueError(f"{name} are {x.dtype}, not 8-bit unsigned")
            if x.dim() != 4:
                raise ValueError(f"{name} are {tuple(x.shape)}, not pages")
            if x.stride(3) != 1 and x.shape[3] > 1:
                raise ValueError(f"the {name} of a slot are not contiguous")
        if scales.shape[:3] != codes.shape[:3] or scales.device != codes.device:
            raise ValueError(f"codes {tuple(codes.shape)} on {codes.device} beside scales "
                             f"{tuple(scales.shape)} on {scales.device}")
        *pages, blocks = scales.shape
        self._bits = codes.shape[3] // (4 * blocks) if blocks else 0
        if self._bits not in (4, 8) or codes.shape[3] != 4 * self._bits * blocks:
            raise ValueError(f"codes of {codes.shape[3]} bytes are not 4 or 8 bits of {blocks} "
                             f"blocks of {BLOCK} elements")
        self._codes, self._scales = codes, scales
        self._n, self._shape = pages[0], (pages[1], pages[2], blocks)
        self._device = codes.get_device() if codes.is_cuda else None
        self._places = codes.data_ptr(), scales.data_ptr()
        self._at = Pages(self._places[0], codes.stride()[:3], self._places[1], scales.stride()[:3])

    codes = property(lambda self: self._codes)
    scales = property(lambda self: self._scales)
    bits = property(lambda self: self._bits)

    def __iter__(self):
        return iter((self._codes, self._scales))

    def __repr__(self):
        n, (heads, size, blocks) = self._n, self._shape
        return (f"MxPages({n} pages of {size} slots, {heads} heads of {blocks} blocks, "
                f"{self._bits} bits)")


def _blocks(head_dim: int) -> int:
    return -(-head_dim // BLOCK)


def new_pages(n_pages: int, kv_heads: int, page_size: int, head_dim: int, bits: int,
              device="cuda") -> MxPages:
    """Pages of zeros."""
    if bits not in (4, 8):
        raise ValueError(f"bits {bits} is neither 4 nor 8")
    if head_dim < 1:
        raise ValueError(f"head_dim {head_dim} is not positive")
    blocks = _blocks(head_dim)
    return MxPages(*(torch.zeros((n_pages, kv_heads, page_size, n), dtype=torch.uint8, device=device)
                     for n in (4 * bits * blocks, blocks)))


def _fits(pages: MxPages, what: str, device: int, n_pages: int, shape) -> Pages:
    """shape: (kv_heads, page_size, blocks)."""
    if (pages._codes.data_ptr(), pages._scales.data_ptr()) != pages._places:
        raise ValueError(f"the tensors of {what} have moved since it was made of them")
    if pages._n < n_pages or pages._shape != shape:
        raise ValueError(f"{what} is {pages}, not at least {n_pages} pages of {shape[1]} slots, "
                         f"{shape[0]} heads of {shape[2]} blocks")
    if pages._device != device:
        _on_gpu(pages._codes, what, device)
    return pages._at


def _caches(k_cache: MxPages, v_cache: MxPages, device: int, n_pages: int, shape):
    shape = shape[0], shape[1], _blocks(shape[2])
    if k_cache._bits != v_cache._bits:
        raise ValueError(f"keys of {k_cache._bits} bits beside values of {v_cache._bits}")
    return (_fits(k_cache, "k_cache", device, n_pages, shape),
            _fits(v_cache, "v_cache", device, n_pages, shape))


def taps_mx_append(k, v, k_cache: MxPages, v_cache: MxPages, plan: PagedPlan, table=None,
                   k_weight=None, eps=1e-6, interleaved=False, stream=None):
    """Writes the new tokens' keys and values into the cache at the plan's places
    (taps_mx_append): keys normed if k_weight is given and rotated by their positions if table is,
    both rounded to the cache's 4 or 8 bits.

    k, v: [tokens, kv_heads, dim] of 16 or 32 bits; k_cache, v_cache: pages of ``new_pages``."""
    device, raw, dtype = _device(), _stream(stream), k.dtype
    code = weight = _dtype(k)
    at, rows, rotary = _table(table, plan.head_dim, device)
    kw = None
    if k_weight is not None:
        kw = _vector(k_weight, "k_weight", plan.head_dim, device, dtype)
        weight = _DTYPES[k_weight.dtype]
    args = AppendArgs(code, weight, rotary, 1 if interleaved else 0, eps, kw, at, rows)
    kc, vc = _caches(k_cache, v_cache, device, plan.n_pages, plan._page_shape)
    _check(load().taps_mx_append(
        C.byref(args), k_cache._bits, *plan.pointers(stream, raw, device),
        _heads(k, "k", device, dtype, plan._k_shape, 3),
        _heads(v, "v", device, dtype, plan._k_shape, 3), kc, vc, raw), "taps_mx_append")


def taps_mx_read(k_cache: MxPages, v_cache: MxPages, slots, head_dim: int, dtype=torch.bfloat16,
                 out=None, stream=None):
    """(k, v) [tokens, kv_heads, head_dim] of the cache's slots (taps_mx_read).

    slots: integers [tokens], page * page_size + slot; one that is no slot of the cache makes its
    token NaN.  dtype: of the results, 16 or 32 bits.  out: (k, v) to fill."""
    device, raw = _device(), _stream(stream)
    if slots.dim() != 1 or not slots.is_contiguous() or \
            slots.dtype not in (torch.int32, torch.int64):
        raise ValueError("slots is not a contiguous vector of integers")
    _on_gpu(slots, "slots", device)
    heads, page_size, _ = k_cache._shape
    n_pages = k_cache._n
    kc, vc = _caches(k_cache, v_cache, device, n_pages, (heads, page_size, head_dim))
    shape = slots.shape[0], heads, head_dim
    if out is None:
        k = _on(stream, lambda: torch.empty(shape, dtype=dtype, device=slots.device))
        v = _on(stream, lambda: _like(k))
        row = heads * head_dim
        kh, vh = Heads(k.data_ptr(), 0, row, head_dim), Heads(v.data_ptr(), 0, row, head_dim)
    else:
        k, v = out
        dtype = k.dtype
        kh, vh = _heads(k, "k", device, dtype, shape, 3), _heads(v, "v", device, dtype, shape, 3)
    args = ReadArgs(_dtype(k), k_cache._bits, shape[0], heads, head_dim, page_size, n_pages,
                    slots.element_size(), slots.data_ptr())
    _check(load().taps_mx_read(C.byref(args), kc, vc, kh, vh, raw), "taps_mx_read")
    return k, v


def taps_mx_attend(q, k_cache: MxPages, v_cache: MxPages, plan: PagedPlan, scale=None, out=None,
                   lse=False, stream=None):
    """Attention of the plan's new tokens over the cache (taps_mx_attend), as
    ``attention.taps_attend`` is over one of 16 bits: q [tokens, q_heads, dim] -> out of the same
    shape; a token that sees no key gets zeros.  scale: dim ** -0.5 unless given.  lse: also
    return [tokens, q_heads] in 32 bits, the log of every row's sum of exponentials (-inf
    without keys)."""
    device, raw, dtype, shape = _device(), _stream(stream), q.dtype, plan._q_shape
    code = _dtype(q)
    qh = _heads(q, "q", device, dtype, shape, 3)
    kc, vc = _caches(k_cache, v_cache, device, plan.n_pages, plan._page_shape)
    n = plan.workspace_bytes
    sums = workspace = None
    given = out
    if out is None:
        out, oh = _on(stream, lambda: _output(q, 3))
    else:
        oh = _heads(out, "out", device, dtype, shape, 3)
    if lse:
        sums = _on(stream, lambda: torch.empty(shape[:2], dtype=torch.float32, device=q.device))
    if n:
        workspace = _on(stream, lambda: torch.empty(n, dtype=torch.uint8, device=q.device))
    _check(load().taps_mx_attend(
        code, k_cache._bits, *plan.pointers(stream, raw, device), qh, kc, vc,
        plan.head_dim ** -0.5 if scale is None else scale, oh,
        None if sums is None else sums.data_ptr(),
        None if workspace is None else workspace.data_ptr(), n, raw), "taps_mx_attend")
    if given is None:
        out, sums = _no_gradient("taps_mx_attend has no gradient", (out, sums), (q,))
    return (out, sums) if lse else out
