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
stream that the call runs on (``stream``, or the current one).  Torch's autograd
follows ``norm_rotate`` alone: a backward pass through the new outputs of another
call raises, as do such calls on inputs with tangents (forward mode); what a call
writes to tensors it is given has no history.
"""
from __future__ import annotations

import ctypes as C
import os
import re
from typing import List

import numpy as np
import torch
from torch.autograd import forward_ad

from . import taps
from .taps import TapsError, _stream   # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtaps_attention.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "taps_attention.h")

BF16, F16, F32 = range(3)
MAX_HEAD_DIM = 256
MAX_ATTEND_DIM = 128
WORKSPACE_PER_ELEMENT = 8192   # bytes of taps_norm_rotate_backward's per element of a head


class Heads(C.Structure):   # stride[3] field by field: made in half the time
    _fields_ = [("data", C.c_void_p), ("stride0", C.c_int64), ("stride1", C.c_int64),
                ("stride2", C.c_int64)]


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
        H = P(Heads)
        L.taps_norm_rotate.argtypes = [P(NormRotateArgs), H, H, H, H, C.c_void_p]
        L.taps_norm_rotate_backward.restype = C.c_int
        L.taps_norm_rotate_backward.argtypes = [P(NormRotateArgs), H, H, H, H, H, H,
                                                C.c_void_p, C.c_void_p, C.c_void_p,
                                                P(C.c_uint64), C.c_void_p]
        L.taps_paged_plan.restype = C.c_int
        L.taps_paged_plan.argtypes = [P(PagedBatch), C.c_uint32, C.c_void_p, P(C.c_uint64),
                                      P(C.c_uint64)]
        L.taps_cache_append.restype = C.c_int
        L.taps_cache_append.argtypes = [P(AppendArgs), C.c_void_p, C.c_void_p, H, H, H, H,
                                        C.c_void_p]
        L.taps_attend.restype = C.c_int
        L.taps_attend.argtypes = [C.c_uint32, C.c_void_p, C.c_void_p, H, H, H, C.c_float, H,
                                  C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
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

# A small call takes less time on the GPU than its marshalling does, so the
# checks are made the short way; one call fetches the device and stream once.

_DTYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}


def _dtype(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"tensors of {t.dtype} are not supported")
    return code


def _device() -> int:
    return torch._C._cuda_getDevice()


def _on_gpu(t, what: str, device: int) -> None:
    if not t.is_cuda:
        raise ValueError(f"{what} is not on the GPU")
    if t.get_device() != device:
        raise ValueError(f"{what} is on {t.device}, not on the current GPU")


def _heads(t, what: str, device: int, dtype, shape, rank: int) -> Heads:
    """A tensor [batch, tokens, heads, dim], or [tokens, heads, dim] as one sequence."""
    if t.dtype is not dtype:
        raise ValueError(f"{what} is {t.dtype}, not {dtype}")
    if t.shape != shape:
        raise ValueError(f"{what} is {tuple(t.shape)}, not {tuple(shape)}")
    _on_gpu(t, what, device)
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: the elements of a head are not contiguous")
    if rank == 3:
        return Heads(t.data_ptr(), 0, s[0], s[1])
    return Heads(t.data_ptr(), s[0], s[1], s[2])



def _vector(w, what: str, dim: int, device: int, dtype) -> int:
    """Pointer to a head's weights."""
    if w.shape != (dim,) or (dim > 1 and w.stride(0) != 1):
        raise ValueError(f"{what} is not a contiguous vector of {dim}")
    if w.dtype is not dtype and w.dtype is not torch.float32:
        raise ValueError(f"{what} is {w.dtype}, neither {dtype} nor 32-bit")
    _on_gpu(w, what, device)
    return w.data_ptr()


def _table(table, dim: int, device: int):
    """(pointer, positions, rotated elements) of a rotation table [positions, 2, rotary / 2]."""
    if table is None:
        return None, 0, 0
    shape = table.shape
    if len(shape) != 3 or shape[1] != 2 or table.dtype is not torch.float32 or \
            not table.is_contiguous():
        raise ValueError("table is not a contiguous 32-bit tensor [positions, 2, pairs]")
    _on_gpu(table, "table", device)
    if 2 * shape[2] > dim:
        raise ValueError(f"table rotates {2 * shape[2]} of {dim} elements")
    return table.data_ptr(), shape[0], 2 * shape[2]


_like = torch.empty_like   # of every way to an output the shortest


def _output(t, rank: int):
    """(a new tensor like ``t``, its Heads).  After overlapping rows (a sliding window over tokens)
    empty_like may not keep a head's elements together."""
    out = _like(t)
    s = out.stride()
    if s[-1] != 1:
        out = torch.empty(t.shape, dtype=t.dtype, device=t.device)
        s = out.stride()
    if rank == 3:
        return out, Heads(out.data_ptr(), 0, s[0], s[1])
    return out, Heads(out.data_ptr(), s[0], s[1], s[2])


_NO_OUTPUT = None, None


def _on(stream, make):
    """New tensors belong to the stream that fills them."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


class _NoGradient(torch.autograd.Function):
    """Hands on the outputs of a call as a function of its inputs that has no gradient."""

    @staticmethod
    def forward(ctx, said, outputs, *inputs):
        ctx.said = said
        return outputs

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(ctx.said)


def _no_gradient(said: str, outputs, inputs):
    """``outputs``, which raise in a backward pass if one of the inputs asks for it: left without
    a history they would pass for constants there.  Raises if an input has a tangent, which has
    no later pass that could."""
    if forward_ad._current_level >= 0:   # unpack_dual asks too, in a third of a microsecond each
        for t in inputs:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise RuntimeError(said)
    if torch.is_grad_enabled():
        for t in inputs:
            if t is not None and t.requires_grad:
                return _NoGradient.apply(said, outputs, *inputs)
    return outputs


def rotation_table(n_positions: int, rotary_dim: int, base: float = 10000.0, device="cuda"):
    """Cosines and sines of position x base^(-2 i / rotary_dim) as a 32-bit tensor
    [n_positions, 2, rotary_dim // 2], angles computed in 64 bits."""
    if rotary_dim < 0 or rotary_dim % 2:
        raise ValueError("rotary_dim is odd or negative")
    inv = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / max(rotary_dim, 1))
    angle = torch.arange(n_positions, dtype=torch.float64)[:, None] * inv
    return torch.stack((angle.cos(), angle.sin()), dim=1).float().to(device)


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------

def _norm_rotate_args(q, k, q_weight, k_weight, table, positions, first, eps, interleaved, device):
    shape = q.shape
    rank = len(shape)
    if rank == 4:
        batch, tokens, q_heads, dim = shape
    elif rank == 3:
        batch, (tokens, q_heads, dim) = 1, shape
    else:
        raise ValueError("q is not [batch, tokens, heads, dim] or [tokens, heads, dim]")
    k_heads = 0
    if k is not None:
        if k.shape[:-2] != shape[:-2] or k.shape[-1] != dim:
            raise ValueError(f"k is {tuple(k.shape)} beside q {tuple(shape)}")
        k_heads = k.shape[-2]
    elif k_weight is not None:
        raise ValueError("k_weight without k")
    dtype = weight = _dtype(q)
    qw = kw = None
    if q_weight is not None:
        qw = _vector(q_weight, "q_weight", dim, device, q.dtype)
        weight = _DTYPES[q_weight.dtype]
    if k_weight is not None:
        kw = _vector(k_weight, "k_weight", dim, device, q.dtype)
        if qw is not None and _DTYPES[k_weight.dtype] != weight:
            raise ValueError("the weights of queries and keys differ in type")
        weight = _DTYPES[k_weight.dtype]
    at, rows, rotary = _table(table, dim, device)
    pos, size = None, 4
    if positions is not None and rotary:
        _on_gpu(positions, "positions", device)
        size = positions.element_size()
        if positions.shape != shape[:-2] or not positions.is_contiguous() or \
                positions.dtype not in (torch.int32, torch.int64):
            raise ValueError(f"positions is not a contiguous integer tensor {tuple(shape[:-2])}")
        pos = positions.data_ptr()
    return NormRotateArgs(batch, tokens, q_heads, k_heads, dim, rotary, dtype, weight,
                          1 if interleaved else 0, eps, qw, kw, at, rows, size, pos, first)


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
    device = _device()
    args = _norm_rotate_args(q, k, q_weight, k_weight, table, positions, first, eps, interleaved,
                             device)
    dtype, shape = q.dtype, q.shape
    rank = len(shape)
    kh = None if k is None else _heads(k, "k", device, dtype, k.shape, rank)
    qh = _heads(q, "q", device, dtype, shape, rank)
    if out is None:   # dense even where q and k are slices of one projection
        (q_out, qoh), (k_out, koh) = _on(
            stream, lambda: (_output(q, rank), _NO_OUTPUT if k is None else _output(k, rank)))
    else:
        q_out, k_out = out
        qoh = _heads(q_out, "out[0]", device, dtype, shape, rank)
        koh = None if k is None else _heads(k_out, "out[1]", device, dtype, k.shape, rank)
    _check(load().taps_norm_rotate(C.byref(args), qh, kh, qoh, koh, _stream(stream)),
           "taps_norm_rotate")
    if out is not None:
        return q_out, k_out
    return _no_gradient("taps_norm_rotate has no gradient: call norm_rotate", (q_out, k_out),
                        (q, k, q_weight, k_weight))


def taps_norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, table, positions=None,
                              first=0, eps=1e-6, interleaved=False, stream=None):
    """(dq, dk, dq_weight, dk_weight): the gradients of ``taps_norm_rotate`` from
    those of its outputs, with its other arguments as they were (None where the
    input is None).  The weights' gradients are summed in 32 bits, in the same
    order every time, and rounded to the weights' type."""
    device = _device()
    args = _norm_rotate_args(q, k, q_weight, k_weight, table, positions, first, eps, interleaved,
                             device)
    dtype, shape = q.dtype, q.shape
    rank = len(shape)
    qh = _heads(q, "q", device, dtype, shape, rank)
    gqh = _heads(dq_out, "dq_out", device, dtype, shape, rank)
    kh = gkh = None
    if k is not None:
        kh = _heads(k, "k", device, dtype, k.shape, rank)
        gkh = _heads(dk_out, "dk_out", device, dtype, k.shape, rank)
    size = WORKSPACE_PER_ELEMENT * shape[-1]

    def make():
        return (_output(q, rank), _NO_OUTPUT if k is None else _output(k, rank),
                None if q_weight is None else _like(q_weight),
                None if k_weight is None else _like(k_weight),
                torch.empty(size, dtype=torch.uint8, device=q.device))
    (dq, dqh), (dk, dkh), dqw, dkw, workspace = _on(stream, make)
    _check(load().taps_norm_rotate_backward(
        C.byref(args), gqh, gkh, qh, kh, dqh, dkh,
        None if dqw is None else dqw.data_ptr(), None if dkw is None else dkw.data_ptr(),
        workspace.data_ptr(), C.byref(C.c_uint64(size)), _stream(stream)),
        "taps_norm_rotate_backward")
    return _no_gradient("taps_norm_rotate_backward has no gradient", (dq, dk, dqw, dkw),
                        (dq_out, dk_out, q, k, q_weight, k_weight))


_function = None


def norm_rotate(q, k, q_weight, k_weight, table, positions=None, first=0, eps=1e-6,
                interleaved=False):
    """``taps_norm_rotate`` for torch's autograd: gradients of q, k and the
    weights come from ``taps_norm_rotate_backward``; they have none of their own."""
    global _function
    if _function is None:
        class NormRotate(torch.autograd.Function):
            @staticmethod
            def forward(ctx, q, k, q_weight, k_weight, table, positions, how):
                ctx.save_for_backward(q, k, q_weight, k_weight, table, positions)
                ctx.how = how
                ctx.set_materialize_grads(False)
                return taps_norm_rotate(q, k, q_weight, k_weight, table, positions, **how)

            @staticmethod
            @torch.autograd.function.once_differentiable
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
            self._at = self._host.data_ptr(), self._gpu.data_ptr()
        self._q_shape = self.tokens, self.q_heads, self.head_dim
        self._k_shape = self.tokens, self.kv_heads, self.head_dim
        self._page_shape = self.kv_heads, self.page_size, self.head_dim

    def pointers(self, stream, raw, device):
        """(host, device) copies, once ``stream`` (its handle: raw) may read the second."""
        if self._gpu is None:
            raise ValueError("the plan was made without a GPU")
        _on_gpu(self._gpu, "plan", device)
        if raw != self._made_on:
            s = torch.cuda.current_stream() if stream is None else stream
            s.wait_event(self._ready)
            self._gpu.record_stream(s)
        return self._at


_units_of = {}


def _units(device) -> int:
    if device not in _units_of:
        _units_of[device] = torch.cuda.get_device_properties(device).multi_processor_count
    return _units_of[device]


def _cache(t, what: str, plan: PagedPlan, device: int, dtype) -> Heads:
    """A cache [pages, kv_heads, page_size, dim] of any strides but the last."""
    shape = t.shape
    if len(shape) != 4 or shape[0] < plan.n_pages or shape[1:] != plan._page_shape:
        raise ValueError(f"{what} is {tuple(shape)}, not at least {plan.n_pages} x "
                         f"{plan._page_shape}")
    return _heads(t, what, device, dtype, shape, 4)


def taps_cache_append(k, v, k_cache, v_cache, plan: PagedPlan, table=None, k_weight=None, eps=1e-6,
                      interleaved=False, stream=None):
    """Writes the new tokens' keys and values into the cache at the plan's
    places (taps_cache_append): keys normed if k_weight is given and rotated by
    their positions if table is, both as in ``taps_norm_rotate``.

    k, v: [tokens, kv_heads, dim]; k_cache, v_cache: [pages, kv_heads,
    page_size, dim]."""
    device, raw, dtype = _device(), _stream(stream), k.dtype
    code = weight = _dtype(k)
    at, rows, rotary = _table(table, plan.head_dim, device)
    kw = None
    if k_weight is not None:
        kw = _vector(k_weight, "k_weight", plan.head_dim, device, dtype)
        weight = _DTYPES[k_weight.dtype]
    args = AppendArgs(code, weight, rotary, 1 if interleaved else 0, eps, kw, at, rows)
    _check(load().taps_cache_append(
        C.byref(args), *plan.pointers(stream, raw, device),
        _heads(k, "k", device, dtype, plan._k_shape, 3),
        _heads(v, "v", device, dtype, plan._k_shape, 3),
        _cache(k_cache, "k_cache", plan, device, dtype),
        _cache(v_cache, "v_cache", plan, device, dtype), raw), "taps_cache_append")


def taps_attend(q, k_cache, v_cache, plan: PagedPlan, scale=None, out=None, lse=False, stream=None):
    """Attention of the plan's new tokens over the cache (taps_attend):
    q [tokens, q_heads, dim] -> out of the same shape; a token that sees no key gets
    zeros.  scale: dim ** -0.5 unless given.  lse: also return [tokens, q_heads]
    in 32 bits, the log of every row's sum of exponentials (-inf without keys)."""
    device, raw, dtype, shape = _device(), _stream(stream), q.dtype, plan._q_shape
    code = _dtype(q)
    qh = _heads(q, "q", device, dtype, shape, 3)
    kh = _cache(k_cache, "k_cache", plan, device, dtype)
    vh = _cache(v_cache, "v_cache", plan, device, dtype)
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
    _check(load().taps_attend(
        code, *plan.pointers(stream, raw, device), qh, kh, vh,
        plan.head_dim ** -0.5 if scale is None else scale, oh,
        None if sums is None else sums.data_ptr(),
        None if workspace is None else workspace.data_ptr(), n, raw), "taps_attend")
    if given is None:
        out, sums = _no_gradient("taps_attend has no gradient", (out, sums), (q, k_cache, v_cache))
    return (out, sums) if lse else out
