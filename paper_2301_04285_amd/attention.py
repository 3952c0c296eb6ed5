"""Python binding of the C ABI in ``include/taps_attention.h`` (ctypes): the
operators that run one device's share of an attention block.

    table = attention.rotation_table(4096, 128)
    plan = attention.PagedPlan(q_lens, kv_lens, pages, n_pages=..., page_size=64,
                               q_heads=32, kv_heads=8, head_dim=128)
    q, _ = attention.taps_norm_rotate(q, None, q_weight, None, table, positions=positions)
    attention.taps_cache_append(k, v, k_cache, v_cache, plan, table=table, k_weight=k_weight)
    out = attention.taps_attend(q, k_cache, v_cache, plan)

Argument marshalling only: every step runs in ``libtaps_attention.so``.  If
the library is missing the calls raise -- there is no other implementation to
fall back to.  Outputs and workspaces come from torch's allocator, on the
stream that the call runs on (``stream``, or the current one).
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import re
from typing import List

import numpy as np

from . import taps
from .taps import TapsError, _stream   # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtaps_attention.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "taps_attention.h")

BF16, F16, F32 = range(3)
MAX_HEAD_DIM = 256
MAX_ATTEND_DIM = 128


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64 * 3)]


class NormRotateArgs(C.Structure):
    _fields_ = [("batch", C.c_uint32), ("tokens", C.c_uint32), ("q_heads", C.c_uint32),
                ("k_heads", C.c_uint32), ("head_dim", C.c_uint32), ("rotary_dim", C.c_uint32),
                ("dtype", C.c_uint32), ("weight_dtype", C.c_uint32), ("interleaved", C.c_uint32),
                ("eps", C.c_float), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p),
                ("table", C.c_void_p), ("n_positions", C.c_uint32),
                ("position_bytes", C.c_uint32), ("positions", C.c_void_p),
                ("first_position", C.c_int64)]


class PagedBatch(C.Structure):
    _fields_ = [("n_seqs", C.c_uint32), ("page_size", C.c_uint32), ("n_pages", C.c_uint32),
                ("pages_stride", C.c_uint32), ("q_lens", C.c_void_p), ("kv_lens", C.c_void_p),
                ("kv_starts", C.c_void_p), ("pages", C.c_void_p), ("q_heads", C.c_uint32),
                ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("causal", C.c_uint32),
                ("window", C.c_uint32)]


class AppendArgs(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("weight_dtype", C.c_uint32), ("rotary_dim", C.c_uint32),
                ("interleaved", C.c_uint32), ("eps", C.c_float), ("k_weight", C.c_void_p),
                ("table", C.c_void_p), ("n_positions", C.c_uint32)]


_lib = None


def load():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2301_04285_amd.build_attention`")
        L = C.CDLL(LIB_PATH)
        P = C.POINTER
        L.taps_norm_rotate.restype = C.c_int
        L.taps_norm_rotate.argtypes = [P(NormRotateArgs), Heads, Heads, Heads, Heads, C.c_void_p]
        L.taps_norm_rotate_backward.restype = C.c_int
        L.taps_norm_rotate_backward.argtypes = [P(NormRotateArgs), Heads, Heads, Heads, Heads,
                                                Heads, Heads, C.c_void_p, C.c_void_p, C.c_void_p,
                                                P(C.c_uint64), C.c_void_p]
        L.taps_paged_plan.restype = C.c_int
        L.taps_paged_plan.argtypes = [P(PagedBatch), C.c_uint32, C.c_void_p, P(C.c_uint64),
                                      P(C.c_uint64)]
        L.taps_cache_append.restype = C.c_int
        L.taps_cache_append.argtypes = [P(AppendArgs), C.c_void_p, C.c_void_p, Heads, Heads, Heads,
                                        Heads, C.c_void_p]
        L.taps_attend.restype = C.c_int
        L.taps_attend.argtypes = [C.c_uint32, C.c_void_p, C.c_void_p, Heads, Heads, Heads,
                                  C.c_float, Heads, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
        L.taps_attention_last_error.restype = C.c_char_p
        L.taps_attention_last_error.argtypes = []
        _lib = L
    return _lib


def declared_symbols() -> List[str]:
    """Entry points declared in include/taps_attention.h."""
    with open(HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"^\s*(?:taps_status|const char \*)\s*(taps_\w+)\s*\(", text,
                                 flags=re.M)))


def last_error() -> str:
    return load().taps_attention_last_error().decode()


def _check(status: int, call: str) -> None:
    if status != taps.OK:
        raise TapsError(status, call, last_error())


# ---------------------------------------------------------------------------
# marshalling
# ---------------------------------------------------------------------------

_DTYPES = {}


def _dtype(t) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32})
    if t.dtype not in _DTYPES:
        raise ValueError(f"tensors of {t.dtype} are not supported")
    return _DTYPES[t.dtype]


def _on_gpu(t, what: str) -> None:
    import torch
    if t.device.type != "cuda":
        raise ValueError(f"{what} is not on the GPU")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what} is on {t.device}, not on the current GPU")


def _heads(t, what: str, like=None, shape=None, rank=4) -> Heads:
    """A tensor [batch, tokens, heads, dim], or [tokens, heads, dim] as one sequence."""
    if like is not None and t.dtype != like.dtype:
        raise ValueError(f"{what} is {t.dtype}, not {like.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} is {tuple(t.shape)}, not {tuple(shape)}")
    _on_gpu(t, what)
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: the elements of a head are not contiguous")
    if rank == 3:
        return Heads(t.data_ptr(), (0, s[0], s[1]))
    return Heads(t.data_ptr(), (s[0], s[1], s[2]))


_NONE = Heads(None, (0, 0, 0))


def _vector(w, what: str, dim: int, like, second=None):
    """(pointer, dtype code) of a head's weights; both weights have one dtype."""
    if w is None:
        return None, None
    if tuple(w.shape) != (dim,) or (dim > 1 and w.stride(0) != 1):
        raise ValueError(f"{what} is not a contiguous vector of {dim}")
    if w.dtype != like.dtype and _dtype(w) != F32:
        raise ValueError(f"{what} is {w.dtype}, neither {like.dtype} nor 32-bit")
    if second is not None and second.dtype != w.dtype:
        raise ValueError("the weights of queries and keys differ in type")
    _on_gpu(w, what)
    return w.data_ptr(), _dtype(w)


def _table(table, dim: int):
    """(pointer, positions, rotated elements) of a rotation table [positions, 2, rotary / 2]."""
    if table is None:
        return None, 0, 0
    if table.dim() != 3 or table.shape[1] != 2 or not table.is_contiguous() or \
            _dtype(table) != F32:
        raise ValueError("table is not a contiguous 32-bit tensor [positions, 2, pairs]")
    _on_gpu(table, "table")
    if 2 * table.shape[2] > dim:
        raise ValueError(f"table rotates {2 * table.shape[2]} of {dim} elements")
    return table.data_ptr(), table.shape[0], 2 * table.shape[2]


def _on(stream):
    """New tensors belong to the stream that fills them."""
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def rotation_table(n_positions: int, rotary_dim: int, base: float = 10000.0, device="cuda"):
    """Cosines and sines of position x base^(-2 i / rotary_dim) as a 32-bit tensor
    [n_positions, 2, rotary_dim // 2], angles computed in 64 bits."""
    import torch
    if rotary_dim < 0 or rotary_dim % 2:
        raise ValueError("rotary_dim is odd or negative")
    inv = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / max(rotary_dim, 1))
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * inv
    return torch.stack((angle.cos(), angle.sin()), dim=1).float().to(device)


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------

def _norm_rotate_args(q, k, q_weight, k_weight, table, positions, first, eps, interleaved):
    if q.dim() not in (3, 4):
        raise ValueError("q is not [batch, tokens, heads, dim] or [tokens, heads, dim]")
    if k is not None and (k.dim() != q.dim() or k.shape[:-2] != q.shape[:-2] or
                          k.shape[-1] != q.shape[-1]):
        raise ValueError(f"k is {tuple(k.shape)} beside q {tuple(q.shape)}")
    if k is None and k_weight is not None:
        raise ValueError("k_weight without k")
    dim = q.shape[-1]
    qw, qt = _vector(q_weight, "q_weight", dim, q, k_weight)
    kw, kt = _vector(k_weight, "k_weight", dim, q)
    at, rows, rotary = _table(table, dim)
    batch, tokens = q.shape[:2] if q.dim() == 4 else (1, q.shape[0])
    pos, size = None, 4
    if positions is not None and rotary:
        _on_gpu(positions, "positions")
        if tuple(positions.shape) != tuple(q.shape[:-2]) or not positions.is_contiguous() or \
                positions.is_floating_point() or positions.element_size() not in (4, 8):
            raise ValueError(f"positions is not a contiguous integer tensor {tuple(q.shape[:-2])}")
        pos, size = positions.data_ptr(), positions.element_size()
    dtype = _dtype(q)
    weight = qt if qt is not None else kt if kt is not None else dtype
    return NormRotateArgs(batch, tokens, q.shape[-2], 0 if k is None else k.shape[-2], dim, rotary,
                          dtype, weight, int(bool(interleaved)), eps, qw, kw, at, rows, size, pos,
                          first)


def taps_norm_rotate(q, k, q_weight, k_weight, table, positions=None, first=0, eps=1e-6,
                     interleaved=False, out=None, stream=None):
    """(q_out, k_out): every head normed by its root mean square and weight,
    then rotated by its token's position (taps_norm_rotate).

    q, k: [batch, tokens, heads, dim] or [tokens, heads, dim], any strides but
    the last; k may be None.  q_weight, k_weight: [dim], or None for no norm.
    table: ``rotation_table`` of the rotated elements, or None for no rotation.
    positions: integers of q's leading dimensions (one that is no row of the
    table makes its token NaN), or None for first, first + 1, ...
    out: (q_out, k_out) to fill; they may be (q, k)."""
    import torch
    args = _norm_rotate_args(q, k, q_weight, k_weight, table, positions, first, eps, interleaved)
    if out is None:
        with _on(stream):
            # dense even where q and k are slices of one projection
            out = (torch.empty(q.shape, dtype=q.dtype, device=q.device),
                   None if k is None else torch.empty(k.shape, dtype=k.dtype, device=k.device))
    q_out, k_out = out
    rank = q.dim()
    none = k is None
    _check(load().taps_norm_rotate(
        C.byref(args), _heads(q, "q", rank=rank), _NONE if none else _heads(k, "k", q, rank=rank),
        _heads(q_out, "out[0]", q, q.shape, rank),
        _NONE if none else _heads(k_out, "out[1]", q, k.shape, rank), _stream(stream)),
        "taps_norm_rotate")
    return q_out, k_out


def taps_norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, table, positions=None,
                              first=0, eps=1e-6, interleaved=False, stream=None):
    """(dq, dk, dq_weight, dk_weight): the gradients of ``taps_norm_rotate`` from
    those of its outputs, with its other arguments as they were (None where the
    input is None).  The weights' gradients are summed in 32 bits, in the same
    order every time, and rounded to the weights' type."""
    import torch
    args = _norm_rotate_args(q, k, q_weight, k_weight, table, positions, first, eps, interleaved)
    rank, none, raw = q.dim(), k is None, _stream(stream)
    need = C.c_uint64()
    L = load()
    _check(L.taps_norm_rotate_backward(C.byref(args), _NONE, _NONE, _NONE, _NONE, _NONE, _NONE,
                                       None, None, None, C.byref(need), raw),
           "taps_norm_rotate_backward")
    with _on(stream):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        dk = None if none else torch.empty(k.shape, dtype=k.dtype, device=k.device)
        dqw = None if q_weight is None else torch.empty_like(q_weight)
        dkw = None if k_weight is None else torch.empty_like(k_weight)
        workspace = torch.empty(need.value, dtype=torch.uint8, device=q.device)
    _check(L.taps_norm_rotate_backward(
        C.byref(args), _heads(dq_out, "dq_out", q, q.shape, rank),
        _NONE if none else _heads(dk_out, "dk_out", q, k.shape, rank), _heads(q, "q", rank=rank),
        _NONE if none else _heads(k, "k", q, rank=rank), _heads(dq, "dq", rank=rank),
        _NONE if none else _heads(dk, "dk", rank=rank),
        None if dqw is None else dqw.data_ptr(), None if dkw is None else dkw.data_ptr(),
        workspace.data_ptr(), C.byref(need), raw), "taps_norm_rotate_backward")
    return dq, dk, dqw, dkw


_function = None


def norm_rotate(q, k, q_weight, k_weight, table, positions=None, first=0, eps=1e-6,
                interleaved=False):
    """``taps_norm_rotate`` for torch's autograd: gradients of q, k and the
    weights come from ``taps_norm_rotate_backward``."""
    global _function
    if _function is None:
        import torch

        class NormRotate(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, q_weight, k_weight, table, positions, how):
                ctx.save_for_backward(q, k, q_weight, k_weight, table, positions)
                ctx.how = how
                ctx.set_materialize_grads(False)
                return taps_norm_rotate(q, k, q_weight, k_weight, table, positions, **how)

            @staticmethod
            def backward(ctx, dq_out, dk_out):
                q, k, q_weight, k_weight, table, positions = ctx.saved_tensors

                def dense(g, x):   # an expanded gradient may have a head of stride 0
                    if x is None:
                        return None
                    if g is None:
                        return torch.zeros_like(x)
                    return g if g.stride(-1) == 1 or x.shape[-1] == 1 else g.contiguous()
                grads = taps_norm_rotate_backward(dense(dq_out, q), dense(dk_out, k), q, k,
                                                  q_weight, k_weight, table, positions, **ctx.how)
                return (*grads, None, None, None)
        _function = NormRotate
    return _function.apply(q, k, q_weight, k_weight, table, positions,
                           {"first": first, "eps": eps, "interleaved": interleaved})


# ---------------------------------------------------------------------------
# the paged cache
# ---------------------------------------------------------------------------

class PagedPlan:
    """One step's sequences laid out for ``taps_cache_append`` and
    ``taps_attend`` (taps_paged_plan), on the host and, in the order of the
    current stream, on the GPU.  One plan serves every layer of the step.

    q_lens[s]: new tokens of sequence s, which lie one after the other in q, k
    and v.  kv_lens[s]: its keys once they are appended.  pages: integers
    [sequences, most pages], the cache page of every page_size keys.
    kv_starts[s]: keys before it do not exist (evicted, padding).  causal: a
    token sees keys up to its own; window > 0: only the last ``window`` of them.
    units: compute units that attention is cut into pieces for (None: the GPU's)."""

    def __init__(self, q_lens, kv_lens, pages, n_pages, page_size, q_heads, kv_heads, head_dim,
                 kv_starts=None, causal=True, window=0, units=None, device="cuda"):
        def ints(x, what, shape=None):
            a = np.asarray(x)
            if a.size and a.dtype.kind not in "iu":
                raise ValueError(f"{what} are not integers")
            if a.size and (a.min() < -2 ** 31 or a.max() >= 2 ** 31):
                raise ValueError(f"{what} exceed 32 bits")
            if shape is not None and a.shape != shape:
                raise ValueError(f"{what} has shape {a.shape}, not {shape}")
            return np.ascontiguousarray(a, dtype=np.int32)
        if min(n_pages, page_size, q_heads, kv_heads, head_dim, window) < 0:
            raise ValueError("a negative size")
        q_lens = ints(q_lens, "q_lens")
        n = q_lens.size
        q_lens = q_lens.reshape(n)
        kv_lens = ints(kv_lens, "kv_lens", (n,))
        pages = ints(pages, "pages")
        if pages.ndim != 2 or pages.shape[0] != n:
            if n:
                raise ValueError(f"pages has shape {pages.shape}, not ({n}, ...)")
            pages = pages.reshape(0, 0)
        starts = None if kv_starts is None else ints(kv_starts, "kv_starts", (n,))
        batch = PagedBatch(n, page_size, n_pages, pages.shape[1], q_lens.ctypes.data,
                           kv_lens.ctypes.data, None if starts is None else starts.ctypes.data,
                           pages.ctypes.data, q_heads, kv_heads, head_dim, int(bool(causal)),
                           min(window, 2 ** 32 - 1))
        self.tokens = int(q_lens.sum(dtype=np.int64))
        self.n_pages, self.page_size = n_pages, page_size
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self._make(batch, units, device)

    def _make(self, batch, units, device) -> None:
        import torch
        size, work = C.c_uint64(), C.c_uint64()
        L = load()
        cus = units or 0
        if device is not None:
            device = torch.device(device)
            if device.index is None:
                device = torch.device(device.type, torch.cuda.current_device())
            cus = cus or _units(device)
        _check(L.taps_paged_plan(C.byref(batch), cus, None, C.byref(size), C.byref(work)),
               "taps_paged_plan")
        self._host = torch.empty(size.value, dtype=torch.uint8, pin_memory=device is not None)
        _check(L.taps_paged_plan(C.byref(batch), cus, self._host.data_ptr(), C.byref(size),
                                 C.byref(work)), "taps_paged_plan")
        self.workspace_bytes = work.value
        self._gpu = self._ready = None
        if device is not None:
            with torch.cuda.device(device):
                self._gpu = self._host.to(device, non_blocking=True)
                self._made_on = _stream(None)
                self._ready = torch.cuda.Event()
                self._ready.record()

    def pointers(self, stream):
        """(host, device) copies, once ``stream`` may read the second."""
        import torch
        if self._gpu is None:
            raise ValueError("the plan was made without a GPU")
        _on_gpu(self._gpu, "plan")
        if _stream(stream) != self._made_on:
            s = torch.cuda.current_stream() if stream is None else stream
            s.wait_event(self._ready)
            self._gpu.record_stream(s)
        return self._host.data_ptr(), self._gpu.data_ptr()


_units_of = {}


def _units(device) -> int:
    import torch
    if device not in _units_of:
        _units_of[device] = torch.cuda.get_device_properties(device).multi_processor_count
    return _units_of[device]


def _cache(t, what: str, plan: PagedPlan, like) -> Heads:
    """A cache [pages, kv_heads, page_size, dim] of any strides but the last."""
    if t.dim() != 4 or t.shape[0] < plan.n_pages or \
            tuple(t.shape[1:]) != (plan.kv_heads, plan.page_size, plan.head_dim):
        raise ValueError(f"{what} is {tuple(t.shape)}, not at least {plan.n_pages} x "
                         f"({plan.kv_heads}, {plan.page_size}, {plan.head_dim})")
    return _heads(t, what, like)


def taps_cache_append(k, v, k_cache, v_cache, plan: PagedPlan, table=None, k_weight=None, eps=1e-6,
                      interleaved=False, stream=None):
    """Writes the new tokens' keys and values into the cache at the plan's
    places (taps_cache_append): keys normed if k_weight is given and rotated by
    their positions if table is, both as in ``taps_norm_rotate``.

    k, v: [tokens, kv_heads, dim]; k_cache, v_cache: [pages, kv_heads,
    page_size, dim]."""
    shape = (plan.tokens, plan.kv_heads, plan.head_dim)
    kw, kt = _vector(k_weight, "k_weight", plan.head_dim, k)
    at, rows, rotary = _table(table, plan.head_dim)
    dtype = _dtype(k)
    args = AppendArgs(dtype, dtype if kt is None else kt, rotary, int(bool(interleaved)), eps, kw,
                      at, rows)
    heads = (_heads(k, "k", k, shape, 3), _heads(v, "v", k, shape, 3),
             _cache(k_cache, "k_cache", plan, k), _cache(v_cache, "v_cache", plan, k))
    _check(load().taps_cache_append(C.byref(args), *plan.pointers(stream), *heads,
                                    _stream(stream)), "taps_cache_append")


def taps_attend(q, k_cache, v_cache, plan: PagedPlan, scale=None, out=None, lse=False, stream=None):
    """Attention of the plan's new tokens over the cache (taps_attend):
    q [tokens, q_heads, dim] -> out of the same shape; a token that sees no key gets
    zeros.  scale: dim ** -0.5 unless given.  lse: also return [tokens, q_heads]
    in 32 bits, the log of every row's sum of exponentials (-inf without keys)."""
    import torch
    shape = (plan.tokens, plan.q_heads, plan.head_dim)
    heads = (_heads(q, "q", q, shape, 3), _cache(k_cache, "k_cache", plan, q),
             _cache(v_cache, "v_cache", plan, q))
    with _on(stream):
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        sums = torch.empty(shape[:2], dtype=torch.float32, device=q.device) if lse else None
        n = plan.workspace_bytes
        workspace = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    _check(load().taps_attend(
        _dtype(q), *plan.pointers(stream), *heads,
        plan.head_dim ** -0.5 if scale is None else scale, _heads(out, "out", q, shape, 3),
        None if sums is None else sums.data_ptr(),
        None if workspace is None else workspace.data_ptr(), n, _stream(stream)), "taps_attend")
    return (out, sums) if lse else out
