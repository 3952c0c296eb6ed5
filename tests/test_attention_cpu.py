"""The attention library without a GPU: exported entry points, plans (which keys
and rows their pieces cover) and refusals of the C ABI."""
import ctypes as C
import math
import random
import subprocess

import numpy as np
import pytest

from paper_2301_04285_amd import attention as A, build_attention, taps
from paper_2301_04285_amd.taps import TapsError


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not os.path.exists(A.LIB_PATH):
        build_attention.build()


def test_declared_entry_points_are_exported():
    exported = subprocess.run(["nm", "-D", "--defined-only", A.LIB_PATH], capture_output=True,
                              text=True, check=True).stdout.split()
    assert A.declared_symbols() == ["taps_attend", "taps_attention_last_error",
                                    "taps_cache_append", "taps_norm_rotate",
                                    "taps_norm_rotate_backward", "taps_paged_plan"]
    assert set(A.declared_symbols()) <= set(exported)


def plan(q_lens, kv_lens, pages=None, page=16, n_pages=None, **kw):
    if pages is None:
        counts = [-(-max(n, 0) // page) for n in kv_lens]
        pages = np.full((len(kv_lens), max(counts + [1])), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(counts):
            pages[s, :n] = range(at, at + n)
            at += n
        n_pages = at if n_pages is None else n_pages
    how = {"q_heads": 8, "kv_heads": 2, "head_dim": 64, "device": None, **kw}
    return A.PagedPlan(q_lens, kv_lens, pages, n_pages=n_pages or 1, page_size=page, **how)


class Header(C.Structure):
    _fields_ = [("magic", C.c_uint32), ("n_seqs", C.c_uint32), ("bytes", C.c_uint64)] + \
        [(n, C.c_uint32) for n in ("tokens", "q_heads", "kv_heads", "head_dim", "page_log2",
                                   "n_pages", "causal", "window", "n_items", "n_joins",
                                   "part_rows", "max_positions", "appendable", "join_rounds",
                                   "n_wide", "reserved")] + [("zeros", C.c_uint32 * 4)] + \
        [(n, C.c_uint64) for n in ("tokens_at", "pages_at", "items_at", "joins_at")]


def parts(p):
    raw = p._host.numpy()
    h = Header.from_buffer_copy(raw[:C.sizeof(Header)].tobytes())

    def words(at, n, k):
        return raw[at:at + 4 * n * k].view(np.int32).reshape(n, k)
    return (h, words(h.tokens_at, h.tokens, 2),
            words(h.items_at, h.n_items, 12), words(h.joins_at, h.n_joins, 8))


@pytest.mark.parametrize("seed", range(75))
def test_plan_covers_every_visible_pair_once(seed):
    """Every row is in one strip; the pieces of a strip follow each other over exactly the keys
    that any of its rows sees; partial results do not overlap and fit the workspace."""
    r = random.Random(seed)
    n = r.randint(1, 5)
    q_lens = [r.choice((0, 1, 1, 2, 7, 40, 300)) for _ in range(n)]
    kv_lens = [r.choice((0, 1, 15, 16, 17, 64, 129, 1000, 5000)) for _ in range(n)]
    if seed >= 60:   # strips of 256 rows
        q_lens, kv_lens = [300] + q_lens, [r.choice((5000, 9001))] + kv_lens
        n += 1
    starts = [r.choice((0, 0, r.randint(0, k))) for k in kv_lens]
    causal = r.random() < 0.8
    window = r.choice((0, 0, 1, 16, 100, 2 ** 31)) if causal else 0
    kv_heads = r.choice((1, 2, 3))
    group = r.choice((1, 3, 4, 16))
    # lengths below the new tokens' leave no tokens to append: plans for attention alone
    p = plan(q_lens, kv_lens, kv_starts=starts, causal=causal, window=window, kv_heads=kv_heads,
             q_heads=group * kv_heads, head_dim=128 if seed >= 60 else 64,
             units=1 + seed % 3 if seed >= 60 else r.choice((1, 16, 256, 100000)))
    h, tokens, items, joins = parts(p)
    assert h.bytes == p._host.numel() and h.tokens == sum(q_lens)
    kinds = items[:, 4].tolist()   # 0: 256 rows, 1: 128, 2: 32
    assert kinds == sorted(kinds) and h.n_wide == kinds.count(0)
    assert list(h.zeros) == [0] * 4
    covered = {}
    used = np.zeros(h.part_rows, dtype=bool)
    for seq, row0, lo, hi, kind, part, *_ in items.tolist():
        rows = min((256, 128, 32)[kind], q_lens[seq] * group - row0)
        assert rows > 0 and row0 % (256, 128, 32)[kind] == 0
        covered.setdefault((seq, row0, rows), []).append((lo, hi, part))
        if part >= 0:
            assert not used[part:part + rows].any() and part + rows <= h.part_rows
            used[part:part + rows] = True
    assert used.all()
    joined = {(s, r0, n): (part, k) for s, r0, n, part, k, *_ in joins.tolist()}
    for s in range(n):
        rows = sorted((a, b) for q, a, b in covered if q == s)
        assert [a for a, _ in rows] == [sum(b for _, b in rows[:i]) for i in range(len(rows))]
        assert sum(b for _, b in rows) == q_lens[s] * group
    for (s, row0, rows), pieces in covered.items():
        pieces.sort()
        lo, hi = pieces[0][0], pieces[-1][1]
        assert all(a[1] == b[0] for a, b in zip(pieces, pieces[1:]))
        seen = set()
        for t in range(row0 // group, (row0 + rows - 1) // group + 1):
            pos = kv_lens[s] - q_lens[s] + t
            last = min(kv_lens[s] - 1, pos) if causal else kv_lens[s] - 1
            first = max(starts[s], pos - window + 1) if window else starts[s]
            seen.update(range(max(0, first), last + 1))
        if seen:
            assert (lo, hi) == (min(seen), max(seen) + 1)
        else:
            assert len(pieces) == 1 and lo >= hi
        if len(pieces) == 1:
            assert pieces[0][2] == -1 and (s, row0, rows) not in joined
        else:
            part, k = joined[s, row0, rows]
            assert k == len(pieces) and [x[2] for x in pieces] == [part + i * rows
                                                                    for i in range(k)]
    assert p.workspace_bytes >= h.part_rows * kv_heads * ((128 if seed >= 60 else 64) * 4 + 8)
    at = 0
    for s in range(n):
        for pos in range(kv_lens[s] - q_lens[s], kv_lens[s]):
            page0 = sum(-(-k // 16) for k in kv_lens[:s])
            slot = -1 if pos < starts[s] else (page0 + pos // 16) * 16 + pos % 16
            assert tokens[at].tolist() == [pos, slot]
            at += 1
    assert h.appendable == all(k >= q for q, k in zip(q_lens, kv_lens))


def test_plan_of_nothing():
    for p in (plan([], []), plan([0, 0], [0, 7])):
        h = parts(p)[0]
        assert h.n_items == 0 and p.workspace_bytes == 0 and p.tokens == 0


@pytest.mark.parametrize("match,args,kw", [
    ("outside 0..2", ([-1], [5]), {}),
    ("outside 0..2", ([1], [-5]), {}),
    ("outside 0..2", ([1], [2 ** 30 + 1]), {"pages": [[0]], "n_pages": 1}),
    ("need 2 pages of 1", ([1], [17]), {"pages": [[0]], "n_pages": 4}),
    ("page 4 outside", ([1], [17]), {"pages": [[0, 4]], "n_pages": 4}),
    ("page -1 outside", ([1], [17]), {"pages": [[-1, 1]], "n_pages": 4}),
    ("written from two places", ([1, 1], [5, 5]), {"pages": [[2], [2]], "n_pages": 4}),
    ("written from two places", ([20], [20]), {"pages": [[2, 2]], "n_pages": 4}),
    ("keys start at", ([1], [5]), {"kv_starts": [6]}),
    ("keys start at", ([1], [5]), {"kv_starts": [-1]}),
    ("power of two", ([1], [5]), {"page": 24}),
    ("power of two", ([1], [5]), {"page": 8}),
    ("power of two", ([1], [5]), {"page": 8192}),
    ("not a multiple", ([1], [5]), {"q_heads": 3}),
    ("not a multiple", ([1], [5]), {"kv_heads": 0}),
    ("head_dim", ([1], [5]), {"head_dim": 0}),
    ("head_dim", ([1], [5]), {"head_dim": 257}),
    ("needs causal", ([1], [5]), {"causal": False, "window": 4}),
    ("2.31 slots", ([1], [5]), {"n_pages": 2 ** 27}),
    ("too many", ([2 ** 30], [5]), {}),
])
def test_plan_refusals(match, args, kw):
    with pytest.raises(TapsError, match=match):
        plan(*args, **kw)


def test_binding_refusals():
    with pytest.raises(ValueError, match="integers"):
        plan([1.5], [5])
    with pytest.raises(ValueError, match="32 bits"):
        plan([1], [5], pages=[[2 ** 31]], n_pages=4)
    with pytest.raises(ValueError, match="shape"):
        plan([1, 1], [5])
    with pytest.raises(ValueError, match="shape"):
        plan([1], [5], pages=[0], n_pages=4)
    with pytest.raises(ValueError, match="shape"):
        plan([1], [5], kv_starts=[0, 0])
    with pytest.raises(ValueError, match="negative"):
        plan([1], [5], window=-1)
    with pytest.raises(ValueError, match="odd"):
        A.rotation_table(4, 3, device="cpu")


def test_pages_may_be_read_twice_and_gone_pages_are_not_looked_at():
    plan([1, 1], [33, 20], pages=[[3, 1, 0], [3, 2, 9]], n_pages=4)      # page 3: a shared prefix
    plan([1, 1], [33, 20], pages=[[-1, 77, 0], [3, 2, -5]], n_pages=4, kv_starts=[32, 0])


def _heads(ptr=0x1000, strides=(512, 512, 64)):
    return A.Heads(ptr, *strides)


def _status(call, *args):
    st = getattr(A.load(), call)(*args)
    return st, A.last_error()


def _args(**kw):
    a = A.NormRotateArgs(1, 4, 8, 0, 64, 64, A.BF16, A.BF16, 0, 1e-6, None, None, 0x1000, 16, 4,
                         None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("match,kw", [
    ("dtype 3", {"dtype": 3}), ("weight_dtype", {"weight_dtype": A.F16}),
    ("head_dim", {"head_dim": 0}), ("head_dim", {"head_dim": 257, "rotary_dim": 0}),
    ("rotary_dim", {"rotary_dim": 63}), ("rotary_dim", {"rotary_dim": 66}),
    ("table is NULL", {"table": None}), ("table is not aligned", {"table": 0x1002}),
    ("eps", {"eps": -1.0}), ("eps", {"eps": math.nan}), ("eps", {"eps": math.inf}),
    ("q_heads", {"q_heads": 0}), ("heads are too many", {"q_heads": 2 ** 21}),
    ("tokens are too many", {"batch": 2 ** 16, "tokens": 2 ** 15}),
    ("position_bytes", {"positions": 0x1000, "position_bytes": 2}),
    ("positions is not aligned", {"positions": 0x1004, "position_bytes": 8}),
    ("exceed the table", {"first_position": 13}), ("exceed the table", {"first_position": -1}),
    ("exceed the table", {"first_position": 2 ** 62}),
])
def test_norm_rotate_refusals(match, kw):
    a = _args(**kw)
    none = A.Heads(None, 0, 0, 0)
    st, said = _status("taps_norm_rotate", C.byref(a), _heads(), none, _heads(), none, None)
    assert st == taps.ERR_ARG and match in said
    need = C.c_uint64()
    st, said = _status("taps_norm_rotate_backward", C.byref(a), _heads(), none, _heads(), none,
                       _heads(), none, None, None, None, C.byref(need), None)
    assert st == taps.ERR_ARG and match in said


def test_pointer_refusals():
    none = A.Heads(None, 0, 0, 0)
    L = A.load()
    assert L.taps_norm_rotate(None, none, none, none, none, None) == taps.ERR_ARG
    a = _args()
    st, said = _status("taps_norm_rotate", C.byref(a), none, none, _heads(), none, None)
    assert st == taps.ERR_ARG and "q is NULL" in said
    st, said = _status("taps_norm_rotate", C.byref(a), _heads(0x1001), none, _heads(), none, None)
    assert st == taps.ERR_ARG and "not aligned" in said
    a = _args(k_heads=2)
    st, said = _status("taps_norm_rotate", C.byref(a), _heads(), _heads(), _heads(), none, None)
    assert st == taps.ERR_ARG and "k_out is NULL" in said
    a = _args(q_weight=0x1000)
    need = C.c_uint64()
    call = [C.byref(a), _heads(), none, _heads(), none, _heads(), none]
    st, _ = _status("taps_norm_rotate_backward", *call, 0x1000, None, None, C.byref(need), None)
    assert st == taps.OK and need.value > 0
    st, said = _status("taps_norm_rotate_backward", *call, None, None, 0x1000, C.byref(need), None)
    assert st == taps.ERR_ARG and "go together" in said
    st, said = _status("taps_norm_rotate_backward", *call, 0x1000, None, 0x1008, C.byref(need), None)
    assert st == taps.ERR_ARG and "16-byte" in said
    less = C.c_uint64(need.value - 1)
    st, said = _status("taps_norm_rotate_backward", *call, 0x1000, None, 0x1000, C.byref(less), None)
    assert st == taps.ERR_CAPACITY and "are needed" in said
    st, said = _status("taps_norm_rotate_backward", *call, 0x1000, None, 0x1000, None, None)
    assert st == taps.ERR_ARG


def test_attend_and_append_refusals():
    p = plan([4], [20])
    host = p._host.data_ptr()
    h = _heads()
    L = A.load()

    def attend(dtype=A.BF16, plan=host, dev=0x1000, q=h, kc=h, vc=h, scale=1.0, out=h, lse=None,
               work=None, n=0):
        return _status("taps_attend", dtype, plan, dev, q, kc, vc, scale, out, lse, work, n, None)
    for match, kw in [("TAPS_BF16", {"dtype": A.F32}), ("NULL", {"plan": None}),
                      ("NULL", {"dev": None}), ("16-byte", {"dev": 0x1008}),
                      ("q is NULL", {"q": A.Heads(None, 0, 0, 0)}),
                      ("v_cache: rows", {"vc": _heads(0x1008)}),
                      ("k_cache: rows", {"kc": _heads(strides=(4, 8, 8))}),
                      ("out: rows", {"out": _heads(strides=(0, 8, 12))}),
                      ("scale", {"scale": 0.0}), ("scale", {"scale": -1.0}),
                      ("scale", {"scale": math.inf}), ("scale", {"scale": math.nan}),
                      ("lse", {"lse": 0x1002})]:
        st, said = attend(**kw)
        assert st == taps.ERR_ARG and match in said, (match, said)
    junk = np.zeros(512, dtype=np.uint8)
    at = junk.ctypes.data + -junk.ctypes.data % 16
    st, said = attend(plan=at)
    assert st == taps.ERR_ARG and "not made by" in said
    split = plan([1], [100000])
    assert split.workspace_bytes > 0
    st, said = attend(plan=split._host.data_ptr())
    assert st == taps.ERR_ARG and "workspace is NULL" in said
    st, said = attend(plan=split._host.data_ptr(), work=0x1000, n=split.workspace_bytes - 1)
    assert st == taps.ERR_CAPACITY
    for dim in (60, 136):
        other = plan([4], [20], head_dim=dim)
        st, said = attend(plan=other._host.data_ptr())
        assert st == taps.ERR_ARG and "multiple of 8" in said

    def append(plan=host, dev=0x1000, k=h, kc=h, **kw):
        a = A.AppendArgs(A.BF16, A.BF16, 64, 0, 1e-6, None, 0x1000, 32)
        for name, v in kw.items():
            setattr(a, name, v)
        return _status("taps_cache_append", C.byref(a), plan, dev, k, h, kc, h, None)
    short = plan([4], [3])
    for match, kw in [("dtype", {"dtype": 9}), ("rotary_dim", {"rotary_dim": 66}),
                      ("table is NULL", {"table": None}), ("eps", {"eps": -1.0}),
                      ("positions up to 20", {"n_positions": 19}),
                      ("k is NULL", {"k": A.Heads(None, 0, 0, 0)}),
                      ("k_cache is not aligned", {"kc": _heads(0x1001)}),
                      ("more new tokens than keys", {"plan": short._host.data_ptr()}),
                      ("NULL", {"plan": None}), ("weight_dtype", {"weight_dtype": A.F16})]:
        st, said = append(**kw)
        assert st == taps.ERR_ARG and match in said, (match, said)
    assert L.taps_cache_append(None, host, 0x1000, h, h, h, h, None) == taps.ERR_ARG


def test_plan_capacity():
    L = A.load()
    one = np.array([1], dtype=np.int32)
    b = A.PagedBatch(1, 16, 4, 1, one.ctypes.data, one.ctypes.data, None,
                     np.zeros(1, dtype=np.int32).ctypes.data, 8, 2, 64, 1, 0)
    pages = np.zeros((1, 1), dtype=np.int32)
    b.pages = pages.ctypes.data
    size, work = C.c_uint64(), C.c_uint64()
    assert L.taps_paged_plan(C.byref(b), 0, None, C.byref(size), C.byref(work)) == taps.OK
    buf = np.full(size.value + 32, 7, dtype=np.uint8)
    at = buf.ctypes.data + -buf.ctypes.data % 16
    less = C.c_uint64(size.value - 1)
    assert L.taps_paged_plan(C.byref(b), 0, at, C.byref(less), C.byref(work)) == taps.ERR_CAPACITY
    assert (buf == 7).all()
    assert L.taps_paged_plan(C.byref(b), 0, at + 8, C.byref(size), C.byref(work)) == taps.ERR_ARG
    assert L.taps_paged_plan(None, 0, None, C.byref(size), C.byref(work)) == taps.ERR_ARG
    assert L.taps_paged_plan(C.byref(b), 0, None, None, C.byref(work)) == taps.ERR_ARG
    b.q_lens = None
    assert L.taps_paged_plan(C.byref(b), 0, None, C.byref(size), C.byref(work)) == taps.ERR_ARG
