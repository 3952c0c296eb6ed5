"""The operators of one device's share of an attention block on the GPU,
against their definitions in 64 bits: types, head layouts, lengths from none to
long, odd sizes, strides, masks that leave rows empty, values in places that
nothing sees."""
import math
import random

import numpy as np
import pytest
import torch

import attention_reference as R
from paper_2301_04285_amd import attention as A
from paper_2301_04285_amd.taps import TapsError

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def say(*a):
    print(*a, flush=True)


def randn(gen, *shape, dtype=BF16, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()


def gen_of(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------

NORM_ROTATE = [
    # batch, tokens, q_heads, k_heads, dim, rotary, interleaved, weights
    (1, 1, 1, 1, 64, 64, False, "both"),
    (3, 5, 4, 2, 128, 128, False, "both"),
    (2, 7, 3, 3, 96, 48, True, "both"),
    (1, 9, 5, 1, 80, 80, True, "both"),
    (2, 3, 33, 2, 64, 32, False, "both"),      # more heads than a workgroup's groups
    (1, 130, 2, 1, 8, 8, False, "both"),       # one lane a row
    (1, 4, 2, 2, 16, 8, True, "both"),
    (1, 4, 2, 2, 24, 8, False, "both"),
    (1, 6, 2, 2, 256, 256, False, "both"),
    (1, 6, 2, 2, 256, 64, True, "none"),
    (2, 5, 2, 1, 36, 36, False, "both"),       # no multiple of 8: element by element
    (1, 5, 2, 1, 7, 6, True, "both"),
    (1, 5, 2, 1, 1, 0, False, "both"),
    (2, 5, 2, 1, 101, 50, False, "both"),
    (1, 5, 3, 2, 254, 254, False, "both"),
    (1, 5, 3, 2, 128, 0, False, "both"),       # norm alone
    (1, 5, 3, 2, 128, 128, False, "none"),     # rotation alone
    (2, 5, 3, 2, 64, 64, False, "q"),
    (2, 5, 3, 2, 64, 64, False, "k"),
    (2, 5, 3, 0, 64, 64, False, "q"),          # queries only
    (1, 0, 3, 2, 64, 64, False, "both"),
]


def _norm_rotate_case(spec, dtype, seed, float_weights=False):
    batch, tokens, q_heads, k_heads, dim, rotary, interleaved, weights = spec
    g = gen_of(seed)
    q = randn(g, batch, tokens, q_heads, dim, dtype=dtype, scale=2)
    k = randn(g, batch, tokens, k_heads, dim, dtype=dtype, scale=2) if k_heads else None
    wt = F32 if float_weights else dtype
    qw = (1 + 0.3 * torch.randn(dim, generator=g)).to(wt).cuda() if weights in ("both", "q") else None
    kw = (1 + 0.3 * torch.randn(dim, generator=g)).to(wt).cuda() \
        if k_heads and weights in ("both", "k") else None
    table = A.rotation_table(300, rotary) if rotary else None
    positions = torch.randint(300, (batch, tokens), generator=g)
    return q, k, qw, kw, table, positions


def _angles(table, positions, batch, tokens):
    if table is None:
        z = np.zeros((batch, tokens, 0))
        return z, z
    rows = R.f64(table)[np.asarray(positions)]
    return rows[..., 0, :], rows[..., 1, :]


def _check_norm_rotate(case, positions, interleaved, run_args, what):
    q, k, qw, kw, table = case
    cos, sin = _angles(table, positions, q.shape[0], q.shape[1])
    outs = A.taps_norm_rotate(q, k, qw, kw, table, eps=EPS, interleaved=interleaved, **run_args)
    g = gen_of(17)
    gs = [None if x is None else randn(g, *x.shape, dtype=x.dtype) for x in (q, k)]
    grads = A.taps_norm_rotate_backward(gs[0], gs[1], q, k, qw, kw, table, eps=EPS,
                                        interleaved=interleaved, **run_args)
    for side, (x, w) in enumerate(((q, qw), (k, kw))):
        if x is None:
            assert outs[side] is None and grads[side] is None and grads[2 + side] is None
            continue
        w64 = None if w is None else R.f64(w)
        y, bound = R.norm_rotate(R.f64(x), w64, cos, sin, interleaved, EPS, x.dtype)
        R.check(outs[side], y, bound, f"{what}: output {side}")
        dx, b, dw, bw = R.norm_rotate_gradients(R.f64(gs[side]), R.f64(x), w64, cos, sin,
                                                interleaved, EPS, x.dtype,
                                                None if w is None else w.dtype)
        R.check(grads[side], dx, b, f"{what}: gradient {side}")
        if w is None:
            assert grads[2 + side] is None
        else:
            R.check(grads[2 + side], dw, bw, f"{what}: weight gradient {side}")


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("spec", NORM_ROTATE)
def test_norm_rotate(spec, dtype):
    q, k, qw, kw, table, positions = _norm_rotate_case(spec, dtype, 3)
    say(f"[gpu] norm_rotate {spec} {dtype}")
    _check_norm_rotate((q, k, qw, kw, table), positions, spec[6],
                       {"positions": positions.int().cuda()}, "positions")
    first = 300 - spec[1]
    consecutive = np.broadcast_to(np.arange(first, 300), spec[:2])
    _check_norm_rotate((q, k, qw, kw, table), consecutive, spec[6], {"first": first}, "first")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_rotate_many_rows(dtype):
    """More tokens than the gradient's workgroups, which then take several each."""
    spec = (3, 700, 2, 1, 64, 64, False, "both")
    q, k, qw, kw, table, positions = _norm_rotate_case(spec, dtype, 5, float_weights=True)
    _check_norm_rotate((q, k, qw, kw, table), positions, False,
                       {"positions": positions.cuda()}, "64-bit positions")


@pytest.mark.parametrize("dim,rotary", [(64, 64), (96, 48), (36, 36)])
def test_norm_rotate_strides(dim, rotary):
    """Slices of one projection, a permuted layout, offsets that only allow single elements,
    a head shared by expansion, and in place."""
    g = gen_of(11)
    table = A.rotation_table(300, rotary)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(BF16).cuda()
    pos = torch.randint(300, (2, 9), generator=g)
    for name, q, k in [
        ("slices", *randn(g, 2, 9, 7, dim).split((4, 3), dim=2)),
        ("permuted", randn(g, 2, 4, 9, dim).transpose(1, 2),
         randn(g, 9, 3, 2, dim).permute(2, 0, 1, 3)),
        ("odd offset", randn(g, 2, 9, 4, dim + 1)[..., 1:], randn(g, 2, 9, 3, dim + 3)[..., :dim]),
        ("expanded", randn(g, 2, 9, 1, dim).expand(2, 9, 4, dim),
         randn(g, 1, 9, 3, dim).expand(2, 9, 3, dim)),
    ]:
        say(f"[gpu] norm_rotate strides {name} {dim}")
        _check_norm_rotate((q, k, w, w, table), pos, False, {"positions": pos.int().cuda()}, name)
    q, k = randn(g, 2, 9, 7, dim).split((4, 3), dim=2)
    want = A.taps_norm_rotate(q, k, w, w, table, positions=pos.int().cuda())
    got = A.taps_norm_rotate(q, k, w, w, table, positions=pos.int().cuda(), out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("interleaved,rotary", [(False, 16), (True, 16), (False, 8), (True, 6)])
def test_norm_rotate_gradient_against_differences(interleaved, rotary):
    """Central differences of a 64-bit forward pass at the kernel's inputs, and the kernel's
    gradient along a direction."""
    g = gen_of(23)
    q, k = randn(g, 1, 3, 2, 16, dtype=F32), randn(g, 1, 3, 1, 16, dtype=F32)
    qw, kw = randn(g, 16, dtype=F32), randn(g, 16, dtype=F32)
    table = A.rotation_table(50, rotary)
    pos = torch.tensor([[3, 49, 17]])
    gs = [randn(g, *x.shape, dtype=F32) for x in (q, k)]
    grads = A.taps_norm_rotate_backward(gs[0], gs[1], q, k, qw, kw, table, eps=EPS,
                                        positions=pos.cuda(), interleaved=interleaved)
    cos, sin = _angles(table, pos, 1, 3)
    x = [R.f64(t) for t in (q, k, qw, kw)]
    rng = np.random.default_rng(4)
    for n in range(4):
        d = rng.standard_normal(x[n].shape)

        def loss(step):
            y = [v + step * d if i == n else v for i, v in enumerate(x)]
            return sum((R.norm_rotate(y[s], y[2 + s], cos, sin, interleaved, EPS, F32)[0] *
                        R.f64(gs[s])).sum() for s in range(2))
        h = 1e-5
        want = (loss(h) - loss(-h)) / (2 * h)
        got = (R.f64(grads[n]) * d).sum()
        # h^2 times third derivatives (1e-10 of values below 1e3), and the 32-bit gradient:
        # 100 roundings' worth of the sum of its terms
        assert abs(got - want) <= 1e-6 + 100 * R.E32 * np.abs(R.f64(grads[n]) * d).sum() + \
            1e-9 * abs(want)


def test_norm_rotate_positions_off_the_table():
    """Such a token is NaN, its neighbours are right."""
    spec = (1, 6, 2, 1, 64, 32, False, "both")
    q, k, qw, kw, table, positions = _norm_rotate_case(spec, BF16, 3)
    pos = torch.tensor([[0, -1, 299, 300, 5, 2 ** 40]])
    good = torch.tensor([0, 2, 4])
    for p in (pos.cuda(), pos.clamp(-7, 2 ** 31 - 1).int().cuda()):
        out, k_out = A.taps_norm_rotate(q, k, qw, kw, table, positions=p)
        dq, dk, dqw, dkw = A.taps_norm_rotate_backward(q, k, q, k, qw, kw, table, positions=p)
        for t in (out, k_out, dq, dk):
            assert t[:, [1, 3, 5]].isnan().all() and t[:, good].isfinite().all()
        assert dqw.isnan().all() and dkw.isnan().all()
        want = A.taps_norm_rotate(q[:, good].contiguous(), k[:, good].contiguous(), qw, kw, table,
                                  positions=pos[:, good].contiguous().cuda())
        assert torch.equal(out[:, good], want[0]) and torch.equal(k_out[:, good], want[1])


def test_norm_rotate_zeros_and_extremes():
    """A row of zeros has gradients from eps; rows with an infinity or a NaN touch no other."""
    g = gen_of(2)
    q = randn(g, 1, 4, 4, 64, dtype=F32)
    q[0, 0, 0] = 0
    q[0, 1, 1, 5] = math.inf
    q[0, 2, 2, 7] = math.nan
    q[0, 3, 3] = 1e15
    w = randn(g, 64, dtype=F32)
    table = A.rotation_table(4, 64)
    out, _ = A.taps_norm_rotate(q, None, w, None, table)
    dq, _, _, _ = A.taps_norm_rotate_backward(q, None, q, None, w, None, table)
    keep = torch.ones(4, 4, dtype=torch.bool)
    keep[1, 1] = keep[2, 2] = False
    assert out[0][keep].isfinite().all() and dq[0][keep].isfinite().all()
    assert (out[0, 0, 0] == 0).all() and out[0, 2, 2].isnan().all()
    cos, sin = _angles(table, np.arange(4)[None], 1, 4)
    x = np.where(keep.numpy()[None, :, :, None], R.f64(q), 0)
    y, bound = R.norm_rotate(x, R.f64(w), cos, sin, False, EPS, F32)
    R.check(np.where(keep.numpy()[None, :, :, None], R.f64(out), 0), y, bound, "kept rows")


def test_norm_rotate_autograd():
    """Through torch's autograd, with an expanded head and an unused output."""
    g = gen_of(9)
    base = randn(g, 2, 5, 1, 64, dtype=F32).requires_grad_()
    k = randn(g, 2, 5, 2, 64, dtype=F32).requires_grad_()
    qw = randn(g, 64, dtype=F32).requires_grad_()
    kw = randn(g, 64, dtype=F32).requires_grad_()
    table = A.rotation_table(64, 64)
    c = randn(g, 2, 5, 3, 64, dtype=F32)
    q_out, k_out = A.norm_rotate(base.expand(2, 5, 3, 64), k, qw, kw, table, first=7)
    (q_out * c).sum().backward()
    grads = A.taps_norm_rotate_backward(c, torch.zeros_like(k), base.detach().expand(2, 5, 3, 64),
                                        k.detach(), qw.detach(), kw.detach(), table, first=7)
    assert torch.equal(base.grad, grads[0].sum(dim=2, keepdim=True))
    assert torch.equal(qw.grad, grads[2])
    assert (k.grad == 0).all() and (kw.grad == 0).all()
    q_out, k_out = A.norm_rotate(base, k, qw, kw, table)
    (q_out.sum() + k_out.sum()).backward()     # gradients of stride 0


def test_norm_rotate_same_every_time():
    spec = (4, 500, 8, 8, 128, 128, False, "both")
    q, k, qw, kw, table, positions = _norm_rotate_case(spec, BF16, 8)
    runs = [A.taps_norm_rotate_backward(q, k, q, k, qw, kw, table, positions=positions.cuda())
            for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))


# ---------------------------------------------------------------------------
# the paged cache
# ---------------------------------------------------------------------------

def page_table(rng, kv_lens, page, spare=1):
    """(pages, n_pages): pages in a random order, -1 where a sequence needs none."""
    counts = [-(-n // page) for n in kv_lens]
    order = list(range(sum(counts) + spare))
    rng.shuffle(order)
    table = np.full((len(kv_lens), max(counts + [1])), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    return table, len(order)


def cache_of(layout, n_pages, kv_heads, page, dim, dtype):
    """A cache full of NaN in one of several layouts, seen as [pages, heads, slots, dim]."""
    shape = {"heads": (n_pages, kv_heads, page, dim), "slots": (n_pages, page, kv_heads, dim),
             "wide": (n_pages, kv_heads, page, 2 * dim),
             "outer": (kv_heads, n_pages, page, dim)}[layout]
    t = torch.full(shape, math.nan, dtype=dtype, device="cuda")
    return {"heads": t, "slots": t.transpose(1, 2), "wide": t[..., dim:],
            "outer": t.transpose(0, 1)}[layout]


APPEND = [
    # new tokens, keys after them, kv_heads, dim, rotary, interleaved, norm, page, layout
    ([1], [1], 1, 64, 64, False, False, 16, "heads"),
    ([1, 1, 1], [16, 17, 500], 8, 128, 128, False, True, 16, "heads"),
    ([40, 0, 7], [40, 0, 300], 2, 96, 48, True, True, 32, "slots"),
    ([3, 0, 130], [3, 9, 131], 3, 80, 80, False, False, 64, "wide"),
    ([5, 20], [5, 70], 2, 36, 18, False, True, 16, "outer"),
    ([5, 20], [5, 70], 1, 7, 0, False, True, 128, "heads"),
    ([5, 20], [5, 70], 2, 256, 256, True, True, 16, "slots"),
    ([4000], [4096], 1, 64, 64, False, True, 4096, "heads"),
    ([0, 0], [0, 5], 2, 64, 64, False, True, 16, "heads"),
]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("spec", APPEND)
def test_append(spec, dtype):
    new, kv, heads, dim, rotary, interleaved, normed, page, layout = spec
    say(f"[gpu] append {spec} {dtype}")
    g = gen_of(6)
    tokens = sum(new)
    k, v = randn(g, tokens, 2 * heads, dim, dtype=dtype, scale=2).split(heads, dim=1)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(dtype).cuda() if normed else None
    table = A.rotation_table(max(kv), rotary) if rotary else None
    pages, n_pages = page_table(random.Random(1), kv, page)
    caches = [cache_of(layout, n_pages, heads, page, dim, dtype) for _ in range(2)]
    plan = A.PagedPlan(new, kv, pages, n_pages=n_pages, page_size=page, q_heads=heads,
                       kv_heads=heads, head_dim=dim)
    A.taps_cache_append(k, v, *caches, plan, table=table, k_weight=w, eps=EPS,
                        interleaved=interleaved)
    left = [R.f64(c) for c in caches]
    at = 0
    for s, (n, m) in enumerate(zip(new, kv)):
        p = np.arange(m - n, m)
        cos, sin = _angles(table, p, n, 0) if table is not None else (np.zeros((n, 0)),) * 2
        y, bound = R.norm_rotate(R.f64(k[at:at + n]), None if w is None else R.f64(w), cos, sin,
                                 interleaved, EPS, dtype)
        for i in range(n):
            place = pages[s, p[i] // page], slice(None), p[i] % page
            R.check(left[0][place], y[i], bound[i], f"key {p[i]} of sequence {s}")
            assert np.array_equal(left[1][place], R.f64(v[at + i]))
            left[0][place] = left[1][place] = math.nan
        at += n
    assert all(np.isnan(c).all() for c in left)   # nothing else was written


ATTEND = [
    # q_lens, kv_lens, q_heads, kv_heads, dim, page, options
    ([1], [1], 1, 1, 64, 16, {}),
    ([1], [1024], 16, 16, 64, 16, {}),
    ([1, 1, 1, 1], [15, 16, 17, 700], 8, 2, 128, 16, {}),
    ([1, 0, 1, 0], [33, 10, 1, 0], 12, 1, 96, 64, {}),
    ([2, 4, 1], [2, 300, 4097], 8, 1, 128, 128, {}),
    ([7, 33, 1], [7, 33, 65], 3, 3, 80, 32, {}),
    ([130], [130], 2, 2, 128, 64, {}),
    ([65, 1, 200], [300, 250, 200], 6, 2, 64, 16, {}),
    ([40], [1500], 8, 2, 128, 64, {}),
    ([300], [300], 1, 1, 40, 16, {}),
    ([129], [129], 4, 4, 8, 16, {}),
    ([5, 3], [5, 77], 64, 1, 64, 16, {}),               # 64 query heads to a key head
    ([1, 1], [900, 40], 8, 2, 128, 64, {"window": 100}),
    ([1, 3], [900, 40], 8, 2, 64, 16, {"window": 1}),
    ([200, 9], [333, 700], 4, 1, 96, 32, {"window": 17}),
    ([300], [1000], 2, 2, 128, 64, {"window": 130}),
    ([64, 2], [64, 90], 4, 2, 64, 16, {"window": 10 ** 9}),
    ([20, 1, 140], [90, 33, 70], 4, 2, 128, 16, {"causal": False}),
    ([20, 3, 2, 170], [5, 0, 1, 90], 4, 2, 64, 16, {}),   # tokens before the first key
    ([20, 1, 100], [90, 33, 170], 4, 2, 128, 16, {"kv_starts": [80, 33, 130]}),
    ([20, 1, 100], [90, 333, 170], 4, 2, 64, 32, {"kv_starts": [17, 300, 60], "window": 40}),
    ([20, 1], [90, 33], 4, 2, 64, 16, {"kv_starts": [11, 30], "causal": False}),
    ([1, 9], [3000, 2600], 8, 2, 128, 64, {"units": 4096}),   # split as far as splits go
    ([1, 200], [3000, 2600], 4, 1, 64, 16, {"units": 4096, "window": 2000}),
    ([140], [2000], 2, 2, 96, 16, {"units": 4096, "causal": False}),
    ([20, 3, 300], [5, 0, 900], 4, 2, 128, 16, {"units": 1}),
    # enough rows for one unit to be worth the largest strips
    ([300, 520], [300, 700], 4, 2, 128, 64, {"units": 1}),
    ([600], [1100], 4, 2, 96, 16, {"units": 1, "window": 130}),
    ([400, 1], [300, 50], 8, 2, 80, 32, {"units": 1}),
    ([700], [90], 4, 2, 64, 16, {"units": 1, "causal": False}),
    ([520, 600], [600, 600], 2, 2, 64, 16, {"units": 1, "kv_starts": [333, 600]}),
    ([260, 257], [260, 321], 4, 4, 128, 16, {"units": 1}),
    ([1030], [2100], 1, 1, 40, 128, {"units": 1, "window": 600}),
]


# enough rows and keys for a few units to be worth strips of 256 rows
WIDE = [
    ([300, 520], [2300, 2700], 4, 2, 128, 64, {"units": 1}),
    ([600], [3100], 4, 2, 96, 16, {"units": 1, "window": 1100}),
    ([400, 1], [2300, 50], 8, 2, 80, 32, {"units": 1}),
    ([700], [1500], 4, 2, 128, 16, {"units": 1, "causal": False}),
    ([520, 600, 300], [6000, 2600, 2600], 8, 2, 72, 16,
     {"units": 1, "kv_starts": [333, 2600, 2590]}),                    # one sequence sees no key
    ([260, 257], [1500, 1321], 4, 4, 128, 16, {"units": 1}),
    ([1030], [2100], 1, 1, 128, 128, {"units": 1}),
    ([200, 300], [150, 2900], 8, 2, 128, 64, {"units": 1}),            # tokens before the first key
    ([300], [9000], 8, 2, 128, 64, {"units": 16}),                     # split over the keys
]


def wide_items(plan):
    return int(plan._host.numpy()[72:76].view(np.int32)[0])   # n_wide of the plan's header


def attend_case(spec, dtype, layout="heads", seed=4):
    """(q, caches, plan, keys and values in 64 bits per sequence); slots that hold no key, or one
    before the sequence's start, hold NaN."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    g = gen_of(seed)
    starts = options.get("kv_starts", [0] * len(kv_lens))
    pages, n_pages = page_table(random.Random(seed), kv_lens, page)
    caches = [cache_of(layout, n_pages, kv_heads, page, dim, dtype) for _ in range(2)]
    kept = []
    for s, n in enumerate(kv_lens):
        k, v = (randn(g, n, kv_heads, dim, dtype=dtype) for _ in range(2))
        j = torch.arange(starts[s], n)
        for c, x in zip(caches, (k, v)):
            c[torch.from_numpy(pages[s]).long()[j // page].cuda(), :, (j % page).cuda()] = \
                x[starts[s]:]
        kept.append((R.f64(k), R.f64(v)))
        pages[s, :starts[s] // page] = -1
    q = randn(g, sum(q_lens), q_heads, dim, dtype=dtype, scale=1.5)
    plan = A.PagedPlan(q_lens, kv_lens, pages, n_pages=n_pages, page_size=page, q_heads=q_heads,
                       kv_heads=kv_heads, head_dim=dim, **options)
    return q, caches, plan, kept


def attend_check(spec, q, kept, out, lse, scale, dtype):
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    starts = options.get("kv_starts", [0] * len(kv_lens))
    at = 0
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        want, bound, w_lse, b_lse = R.attend(
            R.f64(q[at:at + n]), *kept[s], m - n, starts[s], options.get("causal", True),
            options.get("window", 0), scale, dtype)
        R.check(out[at:at + n], want, bound, f"sequence {s}")
        if lse is not None:
            R.check(lse[at:at + n], w_lse, b_lse, f"lse of sequence {s}")
        at += n


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", ATTEND + WIDE)
def test_attend(spec, dtype):
    say(f"[gpu] attend {spec} {dtype}")
    q, caches, plan, kept = attend_case(spec, dtype)
    assert wide_items(plan) or spec not in WIDE
    out, lse = A.taps_attend(q, *caches, plan, lse=True)
    torch.cuda.synchronize()
    attend_check(spec, q, kept, out, lse, spec[4] ** -0.5, dtype)
    assert torch.equal(A.taps_attend(q, *caches, plan), out)   # without lse, and again


@pytest.mark.parametrize("layout", ["slots", "wide", "outer"])
def test_attend_layouts(layout):
    """Caches in other orders, queries and outputs that are slices, a scale of one's own."""
    spec = ([40, 1, 130], [300, 90, 130], 6, 2, 96, 32, {})
    say(f"[gpu] attend layout {layout}")
    q, caches, plan, kept = attend_case(spec, F16, layout)
    wide_q = torch.full((q.shape[0], 9, 104), math.nan, dtype=F16, device="cuda")
    wide_out = torch.full((8, q.shape[0], 96), 3.0, dtype=F16, device="cuda")
    wide_q[:, 2:8, 8:] = q
    out = wide_out[1:7].transpose(0, 1)
    got = A.taps_attend(wide_q[:, 2:8, 8:], *caches, plan, scale=0.31, out=out)
    assert got is out
    attend_check(spec, q, kept, out, None, 0.31, F16)
    assert (wide_out[0] == 3).all() and (wide_out[7] == 3).all()


def test_attend_large_scores():
    """Scores in the hundreds: one key takes all, maxima rise late and in steps."""
    spec = ([130, 1, 3], [600, 2000, 900], 4, 2, 64, 16, {"units": 1024})
    for dtype in (BF16, F16):
        q, caches, plan, kept = attend_case(spec, dtype)
        q = (q * 30).contiguous()
        out, lse = A.taps_attend(q, *caches, plan, lse=True)
        attend_check(spec, q, kept, out, lse, 0.125, dtype)
        rising = [(k * np.linspace(0.02, 1, len(k))[:, None, None], v) for k, v in kept]
        rising = [(R.f64(torch.from_numpy(k).to(dtype)), v) for k, v in rising]
        pages, _ = page_table(random.Random(4), spec[1], spec[5])
        for s, (k, _) in enumerate(rising):
            j = torch.arange(len(k))
            caches[0][torch.from_numpy(pages[s]).long()[j // 16].cuda(), :, (j % 16).cuda()] = \
                torch.from_numpy(k).to(dtype).cuda()
        out, lse = A.taps_attend(q, *caches, plan, lse=True)
        attend_check(spec, q, rising, out, lse, 0.125, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_many_small_numerators(dtype):
    """One key above thousands whose numerators lie below the smallest normal 16-bit numbers, and
    together weigh as much as it does; the key comes first, last or between."""
    n, dim, page = 9000, 64, 64
    g = gen_of(8)
    for q_len, at in ((1, 0), (1, n - 1), (40, 4000), (40, 0)):
        k = torch.zeros(n, 1, dim, dtype=dtype)
        v = torch.randn(n, 1, dim, generator=g).to(dtype)
        q = torch.zeros(q_len, 1, dim, dtype=dtype)
        q[:, 0, 0] = 8.0
        k[:, 0, 0] = -10.75 + 0.25 * torch.randint(0, 3, (n,), generator=g).to(dtype)
        k[at, 0, 0] = 0
        pages, n_pages = page_table(random.Random(2), [n], page)
        caches = [cache_of("heads", n_pages, 1, page, dim, dtype) for _ in range(2)]
        j = torch.arange(n)
        for c, x in zip(caches, (k, v)):
            c[torch.from_numpy(pages[0]).long()[j // page].cuda(), :, (j % page).cuda()] = x.cuda()
        spec = ([q_len], [n], 1, 1, dim, page, {})
        plan = A.PagedPlan([q_len], [n], pages, n_pages=n_pages, page_size=page, q_heads=1,
                           kv_heads=1, head_dim=dim)
        out, lse = A.taps_attend(q.cuda(), *caches, plan, lse=True)   # scale 1/8: scores as in k
        attend_check(spec, q, [(R.f64(k), R.f64(v))], out, lse, 0.125, dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", [
    ([4, 30], [4, 200], 4, 2, 128, 16, {}),                  # few rows, several tokens
    ([70, 3], [70, 90], 2, 2, 64, 16, {"window": 20}),
    ([140], [500], 2, 1, 96, 32, {"window": 65}),
    ([300], [330], 4, 2, 128, 64, {"units": 1}),
    ([300], [700], 4, 2, 80, 16, {"units": 1, "window": 100}),
    ([40], [1500], 8, 2, 128, 64, {"units": 4096}),
    ([300], [1700], 4, 2, 128, 64, {"units": 1}),            # 256 rows an item
    ([300], [2900], 4, 2, 80, 16, {"units": 1, "window": 1500}),
])
def test_attend_infinities_and_nans(spec, dtype):
    """Keys and values that are infinite or NaN, among the new tokens and before: they reach the
    tokens that see them and no others."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    say(f"[gpu] attend infinities {spec} {dtype}")
    q, caches, plan, kept = attend_case(spec, dtype)
    pages, _ = page_table(random.Random(4), kv_lens, page)
    rng = random.Random(5)
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for which, value in ((1, math.nan), (1, math.inf), (1, -math.inf), (0, math.nan)):
            j = m - 1 - rng.randrange(min(m, n + 40))   # a new token, or one just before them
            h, d = rng.randrange(kv_heads), rng.randrange(dim)
            caches[which][pages[s, j // page], h, j % page, d] = value
            kept[s][which][j, h, d] = value
    out, lse = A.taps_attend(q, *caches, plan, lse=True)
    want_bad = clean = 0
    at = 0
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        with np.errstate(invalid="ignore"):
            want, bound, _, _ = R.attend(R.f64(q[at:at + n]), *kept[s], m - n, 0, True,
                                         options.get("window", 0), dim ** -0.5, dtype)
        got = R.f64(out[at:at + n])
        bad = ~np.isfinite(want)
        assert np.array_equal(bad, ~np.isfinite(got)), "not the same outputs are finite"
        R.check(np.where(bad, 0, got), np.where(bad, 0, want), np.where(bad, 1, bound), "finite")
        inf = np.isinf(want) & ~np.isnan(got)
        assert np.array_equal(got[inf], want[inf])
        want_bad, clean = want_bad + bad.sum(), clean + (~bad).sum()
        at += n
    assert want_bad and clean


def test_attend_far_offsets():
    """Caches of more than 2^32 bytes and 2^31 elements, a sequence at their far end."""
    page, heads, dim, n_pages = 64, 8, 128, 40000   # 2.6e9 elements, 5.2e9 bytes each
    g = gen_of(1)
    caches = [torch.empty((n_pages, heads, page, dim), dtype=BF16, device="cuda") for _ in range(2)]
    kv = [200, 150]
    pages = np.array([[39999, 3, 39997, 32769], [39990, 39991, 5, -1]], dtype=np.int32)
    kept = []
    for s, n in enumerate(kv):
        k, v = (randn(g, n, heads, dim) for _ in range(2))
        j = torch.arange(n)
        for c, x in zip(caches, (k, v)):
            c[torch.from_numpy(pages[s]).long()[j // page].cuda(), :, (j % page).cuda()] = x
        kept.append((R.f64(k), R.f64(v)))
    spec = ([1, 40], kv, 8, 8, 128, page, {})
    plan = A.PagedPlan([1, 40], kv, pages, n_pages=n_pages, page_size=page, q_heads=8, kv_heads=8,
                       head_dim=128)
    q = randn(g, 41, 8, 128)
    out = A.taps_attend(q, *caches, plan)
    attend_check(spec, q, kept, out, None, 128 ** -0.5, BF16)
    k, v = randn(g, 41, 8, 128), randn(g, 41, 8, 128)
    A.taps_cache_append(k, v, *caches, plan)
    assert torch.equal(caches[0][32769, :, 7], k[0]) and torch.equal(caches[1][5, :, 21], v[40])


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def _step(dtype=BF16):
    """A decoding step's tensors: q, k, v, weights, table, pages."""
    g = gen_of(12)
    kv = [70, 1, 333, 128]
    pages, n_pages = page_table(random.Random(3), kv, 16)
    caches = [torch.zeros((n_pages, 2, 16, 64), dtype=dtype, device="cuda") for _ in range(2)]
    for c in caches:
        c.copy_(randn(g, *c.shape, dtype=dtype))
    plan = A.PagedPlan([1] * 4, kv, pages, n_pages=n_pages, page_size=16, q_heads=8, kv_heads=2,
                       head_dim=64)
    qkv = randn(g, 4, 12, 64, dtype=dtype, scale=2)
    w = randn(g, 64, dtype=dtype)
    table = A.rotation_table(400, 64)
    positions = torch.tensor(kv, dtype=torch.int32).cuda() - 1
    return qkv, w, table, positions, caches, plan


def _run_step(qkv, w, table, positions, caches, plan, **kw):
    q, k, v = qkv.split((8, 2, 2), dim=1)
    q, _ = A.taps_norm_rotate(q, None, w, None, table, positions=positions, **kw)
    A.taps_cache_append(k, v, *caches, plan, table=table, k_weight=w, **kw)
    return A.taps_attend(q, *caches, plan, **kw)


def test_step_agrees_with_its_parts():
    """The appended keys are the rotated keys of norm_rotate, bit for bit."""
    qkv, w, table, positions, caches, plan = _step()
    _run_step(qkv, w, table, positions, caches, plan)
    q, k, v = qkv.split((8, 2, 2), dim=1)
    _, kr = A.taps_norm_rotate(q, k, w, w, table, positions=positions)
    pages, _ = page_table(random.Random(3), [70, 1, 333, 128], 16)
    for s, n in enumerate([70, 1, 333, 128]):
        place = pages[s, (n - 1) // 16], slice(None), (n - 1) % 16
        assert torch.equal(caches[0][place], kr[s]) and torch.equal(caches[1][place], v[s])


def test_step_in_a_graph():
    """Captured once, replayed with other inputs between eager work."""
    qkv, w, table, positions, caches, plan = _step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run_step(qkv, w, table, positions, caches, plan)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _run_step(qkv, w, table, positions, caches, plan)
    g = gen_of(30)
    for _ in range(4):
        qkv.copy_(randn(g, *qkv.shape, scale=2))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = _run_step(qkv, w, table, positions, caches, plan)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_step_on_another_stream():
    """The stream argument, while the current stream is busy with other memory."""
    qkv, w, table, positions, caches, plan = _step()
    want = _run_step(qkv, w, table, positions, caches, plan)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        noise = [torch.full((1 << 20,), math.nan, device="cuda") for _ in range(4)]
        side.wait_stream(torch.cuda.current_stream())
        got = _run_step(qkv, w, table, positions, caches, plan, stream=side)
        del noise
        torch.full((1 << 20,), math.nan, device="cuda")
        side.synchronize()
        assert torch.equal(got, want)


def test_gpu_refusals():
    q = torch.zeros(4, 8, 64, dtype=BF16, device="cuda")
    table = A.rotation_table(16, 64)
    w = torch.ones(64, dtype=BF16, device="cuda")
    with pytest.raises(TapsError, match="exceed the table"):
        A.taps_norm_rotate(q, None, w, None, table, first=13)
    with pytest.raises(TapsError, match="exceed the table"):
        A.taps_norm_rotate(q, None, w, None, table, first=-1)
    with pytest.raises(TapsError, match="eps"):
        A.taps_norm_rotate(q, None, w, None, table, eps=-1.0)
    with pytest.raises(TapsError, match="head_dim"):
        A.taps_norm_rotate(torch.zeros(2, 1, 300, device="cuda"), None, None, None, None)
    with pytest.raises(ValueError, match="contiguous"):
        A.taps_norm_rotate(q.transpose(1, 2), None, None, None, None)
    with pytest.raises(ValueError, match="q_weight"):
        A.taps_norm_rotate(q, None, w[:32], None, table)
    with pytest.raises(ValueError, match="not on the GPU"):
        A.taps_norm_rotate(q.cpu(), None, None, None, None)
    with pytest.raises(ValueError, match="positions"):
        A.taps_norm_rotate(q, None, w, None, table, positions=torch.zeros(3, device="cuda").int())
    with pytest.raises(ValueError, match="not supported"):
        A.taps_norm_rotate(q.double(), None, None, None, None)
    cache = torch.zeros(2, 8, 16, 64, dtype=BF16, device="cuda")
    plan = A.PagedPlan([4], [20], [[0, 1]], n_pages=2, page_size=16, q_heads=8, kv_heads=8,
                       head_dim=64)
    with pytest.raises(TapsError, match="positions up to 20"):
        A.taps_cache_append(q, q, cache, cache.clone(), plan, table=table)
    with pytest.raises(ValueError, match="k_cache"):
        A.taps_cache_append(q, q, cache[:1], cache, plan)
    with pytest.raises(ValueError, match="is torch.float16"):
        A.taps_cache_append(q, q.half(), cache, cache, plan)
    with pytest.raises(ValueError, match="q is"):
        A.taps_attend(q[:3], cache, cache, plan)
    with pytest.raises(TapsError, match="scale"):
        A.taps_attend(q, cache, cache, plan, scale=0.0)
    with pytest.raises(TapsError, match="scale"):
        A.taps_attend(q, cache, cache, plan, scale=math.nan)
    with pytest.raises(TapsError, match="neither TAPS_BF16"):
        A.taps_attend(q.float(), cache.float(), cache.float(), plan)
    odd = torch.zeros(4 * 8 * 64 + 1, dtype=BF16, device="cuda")[1:].view(4, 8, 64)
    with pytest.raises(TapsError, match="16 bytes"):
        A.taps_attend(odd, cache, cache, plan)
    short = A.PagedPlan([4], [3], [[0]], n_pages=2, page_size=16, q_heads=8, kv_heads=8, head_dim=64)
    with pytest.raises(TapsError, match="more new tokens than keys"):
        A.taps_cache_append(q, q, cache, cache, short)
    host = A.PagedPlan([4], [20], [[0, 1]], n_pages=2, page_size=16, q_heads=8, kv_heads=8,
                       head_dim=64, device=None)
    with pytest.raises(ValueError, match="without a GPU"):
        A.taps_attend(q, cache, cache, host)
