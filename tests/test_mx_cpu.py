"""The cache in microscaling formats without a GPU: exported entry points, refusals of the C ABI
and of the binding, and the reference's own codes."""
import ctypes as C
import math
import subprocess

import numpy as np
import pytest
import torch

import mx_reference as M
from paper_2301_04285_amd import attention as A, build_attention, mx, taps
from test_attention_cpu import plan


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not os.path.exists(A.LIB_PATH):
        build_attention.build()


def test_declared_entry_points_are_exported():
    exported = subprocess.run(["nm", "-D", "--defined-only", A.LIB_PATH], capture_output=True,
                              text=True, check=True).stdout.split()
    assert mx.declared_symbols() == ["taps_mx_append", "taps_mx_attend", "taps_mx_read"]
    assert set(mx.declared_symbols()) <= set(exported)


def _heads(ptr=0x1000, strides=(512, 512, 64)):
    return A.Heads(ptr, *strides)


def _pages(codes=0x1000, code_strides=(1024, 512, 32), scales=0x1001, scale_strides=(32, 32, 2)):
    return mx.Pages(codes, code_strides, scales, scale_strides)


def _status(call, *args):
    st = getattr(mx.load(), call)(*args)
    return st, A.last_error()


PAGES = [
    ("is NULL", {"codes": None}), ("is NULL", {"scales": None}),
    ("multiples of 16", {"codes": 0x1008}), ("multiples of 16", {"code_strides": (1000, 512, 32)}),
    ("multiples of 16", {"code_strides": (1024, 40, 32)}),
    ("multiples of 16", {"code_strides": (1024, 512, 40)}),
    ("2.27 bytes", {"code_strides": (1024, 512, 2 ** 27)}),
    ("2.27 bytes", {"code_strides": (1024, 512, -32)}),
    ("2.27 bytes", {"scale_strides": (32, 32, 2 ** 27)}),
]


def test_append_refusals():
    p, short = plan([4], [20]), plan([4], [3])

    def append(plan=p, dev=0x1000, bits=4, k=_heads(), v=_heads(), kc=_pages(), vc=_pages(), **kw):
        a = A.AppendArgs(A.BF16, A.BF16, 64, 0, 1e-6, None, 0x1000, 32)
        for name, x in kw.items():
            setattr(a, name, x)
        return _status("taps_mx_append", C.byref(a), bits, plan and plan._host.data_ptr(), dev, k, v,
                       kc, vc, None)
    for match, kw in [("bits 5", {"bits": 5}), ("dtype", {"dtype": 9}), ("NULL", {"plan": None}),
                      ("NULL", {"dev": None}), ("rotary_dim", {"rotary_dim": 66}),
                      ("table is NULL", {"table": None}), ("eps", {"eps": -1.0}),
                      ("eps", {"eps": math.inf}), ("weight_dtype", {"weight_dtype": A.F16}),
                      ("k_weight is not aligned", {"k_weight": 0x1001}),
                      ("positions up to 20", {"n_positions": 19}),
                      ("k is NULL", {"k": _heads(None)}), ("v is not aligned", {"v": _heads(0x1001)}),
                      ("more new tokens than keys", {"plan": short}),
                      ("multiple of 8", {"plan": plan([4], [20], head_dim=60)}),
                      ("multiple of 8", {"plan": plan([4], [20], head_dim=136)})]:
        st, said = append(**kw)
        assert st == taps.ERR_ARG and match in said, (match, said)
    for match, kw in PAGES:
        for side in ("kc", "vc"):
            st, said = append(**{side: _pages(**kw)})
            assert st == taps.ERR_ARG and said.startswith(side[0] + "_cache"), (match, said)
    assert append(kc=None)[0] == taps.ERR_ARG
    assert mx.load().taps_mx_append(None, 4, p._host.data_ptr(), 0x1000, _heads(), _heads(),
                                    _pages(), _pages(), None) == taps.ERR_ARG
    assert append(plan=plan([0], [20]))[0] == taps.OK   # nothing to append


def test_attend_refusals():
    p = plan([4], [20])

    def attend(dtype=A.BF16, bits=8, plan=p, dev=0x1000, q=_heads(), kc=_pages(), vc=_pages(),
               scale=1.0, out=_heads(), lse=None, work=None, n=0):
        return _status("taps_mx_attend", dtype, bits, plan and plan._host.data_ptr(), dev, q, kc, vc,
                       scale, out, lse, work, n, None)
    for match, kw in [("TAPS_BF16", {"dtype": A.F32}), ("bits 16", {"bits": 16}),
                      ("NULL", {"plan": None}), ("NULL", {"dev": None}),
                      ("16-byte", {"dev": 0x1008}), ("q is NULL", {"q": _heads(None)}),
                      ("q: rows", {"q": _heads(0x1008)}),
                      ("out: rows", {"out": _heads(strides=(0, 8, 12))}),
                      ("scale", {"scale": 0.0}), ("scale", {"scale": math.nan}),
                      ("lse", {"lse": 0x1002}),
                      ("multiple of 8", {"plan": plan([4], [20], head_dim=60)}),
                      ("multiple of 8", {"plan": plan([4], [20], head_dim=136)})]:
        st, said = attend(**kw)
        assert st == taps.ERR_ARG and match in said, (match, said)
    for match, kw in PAGES:
        for side in ("kc", "vc"):
            st, said = attend(**{side: _pages(**kw)})
            assert st == taps.ERR_ARG and said.startswith(side[0] + "_cache"), (match, said)
    split = plan([1], [100000])
    assert attend(plan=split)[0] == taps.ERR_ARG
    assert attend(plan=split, work=0x1000, n=split.workspace_bytes - 1)[0] == taps.ERR_CAPACITY
    assert attend(plan=split, work=0x1008, n=split.workspace_bytes)[0] == taps.ERR_ARG
    assert attend(plan=plan([0], [20]))[0] == taps.OK


def test_read_refusals():
    def read(k=_heads(), v=_heads(), kc=_pages(), vc=_pages(), **kw):
        a = mx.ReadArgs(A.BF16, 4, 10, 2, 64, 16, 4, 4, 0x1000)
        for name, x in kw.items():
            setattr(a, name, x)
        return _status("taps_mx_read", C.byref(a), kc, vc, k, v, None)
    for match, kw in [("dtype 3", {"dtype": 3}), ("bits 0", {"bits": 0}),
                      ("multiple of 8", {"head_dim": 0}), ("multiple of 8", {"head_dim": 12}),
                      ("multiple of 8", {"head_dim": 256}), ("power of two", {"page_size": 24}),
                      ("power of two", {"page_size": 8}), ("power of two", {"page_size": 8192}),
                      ("kv_heads", {"kv_heads": 0}), ("kv_heads", {"kv_heads": 65536}),
                      ("too many", {"tokens": 2 ** 31}), ("slot_bytes", {"slot_bytes": 2}),
                      ("slots is NULL", {"slots": None}),
                      ("slots is not aligned", {"slots": 0x1004, "slot_bytes": 8}),
                      ("no pages", {"n_pages": 0}), ("k is NULL", {"k": _heads(None)}),
                      ("v is not aligned", {"v": _heads(0x1001)})]:
        st, said = read(**kw)
        assert st == taps.ERR_ARG and match in said, (match, said)
    for match, kw in PAGES:
        for side in ("kc", "vc"):
            st, said = read(**{side: _pages(**kw)})
            assert st == taps.ERR_ARG and said.startswith(side[0] + "_cache"), (match, said)
    assert mx.load().taps_mx_read(None, _pages(), _pages(), _heads(), _heads(), None) == taps.ERR_ARG
    assert read(tokens=0, slots=None)[0] == taps.OK


def test_pages():
    for dim, bits, codes, scales in ((128, 4, 64, 4), (96, 8, 96, 3), (40, 4, 32, 2), (8, 8, 32, 1)):
        c = mx.new_pages(3, 2, 16, dim, bits, device="cpu")
        assert c.codes.shape == (3, 2, 16, codes) and c.scales.shape == (3, 2, 16, scales)
        assert c.bits == bits and not c.codes.any() and not c.scales.any()
    with pytest.raises(ValueError, match="neither 4 nor 8"):
        mx.new_pages(3, 2, 16, 64, 5, device="cpu")
    with pytest.raises(ValueError, match="not positive"):
        mx.new_pages(3, 2, 16, 0, 4, device="cpu")


def test_pages_refusals():
    def zeros(*shape, dtype=torch.uint8):
        return torch.zeros(shape, dtype=dtype)
    codes, scales = zeros(3, 2, 16, 64), zeros(3, 2, 16, 4)
    for match, c, s in [("codes are torch.int8", codes.char(), scales),
                        ("scales are torch.float32", codes, scales.float()),
                        ("not pages", codes[0], scales), ("not pages", codes, scales[0]),
                        ("codes of a slot", zeros(3, 2, 64, 16).transpose(2, 3), scales),
                        ("scales of a slot", codes, zeros(3, 2, 4, 16).transpose(2, 3)),
                        ("beside scales", codes, scales[:2]), ("beside scales", codes[:, :1], scales),
                        ("beside scales", codes[:, :, :8], scales),
                        ("not 4 or 8 bits", codes[..., :48], scales),
                        ("not 4 or 8 bits", codes[..., :63], scales[..., :3]),
                        ("not 4 or 8 bits", codes, scales[..., :0])]:
        with pytest.raises(ValueError, match=match):
            mx.MxPages(c, s)


def test_pages_stay_with_their_tensors():
    """What was looked at once is what later calls write to: neither tensor can be put in the
    place of another, and calls refuse pages whose tensors have moved."""
    c = mx.new_pages(3, 2, 16, 128, 4, device="cpu")
    for name in ("codes", "scales", "bits"):
        x = getattr(c, name)
        with pytest.raises(AttributeError):
            setattr(c, name, x if name == "bits" else x.clone())
        assert getattr(c, name) is x
    fits = None, 3, (2, 16, 4)   # a device that is that of CPU tensors
    c.codes.fill_(3)
    c.scales[1] = 9
    assert mx._fits(c, "k_cache", *fits) is c._at and c._at.codes == c.codes.data_ptr()

    def grown(x):
        x.resize_(9, *x.shape[1:])

    def replaced(x):
        x.set_(torch.zeros_like(x))

    def given_data(x):
        x.data = torch.zeros_like(x)

    def freed(x):
        x.untyped_storage().resize_(0)
    for move in (grown, replaced, given_data, freed):
        for name in ("codes", "scales"):
            c = mx.new_pages(3, 2, 16, 128, 4, device="cpu")
            held = c.codes.clone(), c.scales.clone()   # so that a new place is another one
            move(getattr(c, name))
            with pytest.raises(ValueError, match="k_cache have moved"):
                mx._fits(c, "k_cache", *fits)
            del held


@pytest.mark.parametrize("bits", [4, 8])
def test_reference_codes(bits):
    """Every number that a code stands for is held as it is; others move to a neighbour that no
    other is nearer than; the scale is the smallest that takes the largest."""
    sizes = M.SIZES[bits]
    for e in (-100, -3, 0, 7):
        x = np.zeros((len(sizes), 32))
        x[:, 0], x[:, 1], x[:, 2] = sizes[-1], sizes, -sizes
        codes, scales = M.encode(x * 2.0 ** e, bits, torch.float32)
        assert (scales == e + 127).all()
        assert np.array_equal(M.decode(codes, scales, 32), x * 2.0 ** e)
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((200, 64)) * np.exp(rng.standard_normal((200, 1)))).astype(np.float32)
    codes, scales = M.encode(x, bits, torch.float32)
    back = M.decode(codes, scales, 64)
    scale = 2.0 ** (scales.astype(int) - 127)
    top = np.abs(x).reshape(200, 2, 32).max(axis=-1)
    assert (top <= M.LIMIT[bits] * scale).all() and (top > M.LIMIT[bits] * scale / 2).all()
    grid = np.concatenate([-sizes, sizes])
    every = np.abs(x[..., None] - grid * np.repeat(scale, 32, axis=-1)[..., None]).min(axis=-1)
    assert np.array_equal(np.abs(x - back), every)
    # as the ABI says
    at = np.abs(x) / np.repeat(scale, 32, axis=-1)
    step = np.where(at < 2, 0.25, np.where(at < 4, 0.5, 1)) if bits == 4 else \
        np.maximum(at * 2.0 ** -4, 2.0 ** -10)
    assert (np.abs(x - back) <= step * np.repeat(scale, 32, axis=-1)).all()
