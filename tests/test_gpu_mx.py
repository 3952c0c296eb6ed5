"""The cache in microscaling formats on the GPU: codes and scales bit for bit, slots read
back, attention over it against its definition in 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

import attention_reference as R
import mx_reference as M
from paper_2301_04285_amd import attention as A, mx
from paper_2301_04285_amd.taps import TapsError
from test_gpu_attention import ATTEND, WIDE, attend_check, gen_of, page_table, randn, say, wide_items

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def pages_of(layout, n_pages, heads, page, dim, bits, fill):
    """Pages whose bytes are all ``fill``, in some order of the axes."""
    blocks = -(-dim // 32)
    made = []
    for size in (4 * bits * blocks, blocks):
        if layout == "heads":
            t = torch.full((n_pages, heads, page, size), fill, dtype=torch.uint8, device="cuda")
        elif layout == "slots":   # a slot's heads side by side
            t = torch.full((n_pages, page, heads, size), fill, dtype=torch.uint8,
                           device="cuda").transpose(1, 2)
        else:                     # a slice of wider rows
            t = torch.full((heads, n_pages, page, size + 16), fill, dtype=torch.uint8,
                           device="cuda").transpose(0, 1)[..., 16:]
        made.append(t)
    return mx.MxPages(*made)


def host(t):
    return t.cpu().numpy()


def set_keys(pages, table, s, x, page, first=0):
    """x [keys, heads, dim] in 64 bits becomes keys first .. of sequence s; their values in 64
    bits."""
    codes, scales = M.encode(x, pages.bits, BF16)
    j = torch.arange(first, first + len(x))
    at = torch.from_numpy(table[s]).long()[j // page].cuda(), slice(None), (j % page).cuda()
    pages.codes[at] = torch.from_numpy(codes).cuda()
    pages.scales[at] = torch.from_numpy(scales).cuda()
    return M.decode(codes, scales, x.shape[-1])


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

APPEND = [
    # new tokens, keys after them, heads, dim, rotary, interleaved, normed, page, layout
    ([1, 1, 1], [1, 17, 40], 2, 64, 64, False, True, 16, "heads"),
    ([5, 0, 20], [9, 0, 20], 3, 128, 128, False, True, 16, "slots"),
    ([40], [133], 2, 96, 48, True, True, 64, "wide"),
    ([33, 2], [33, 200], 1, 80, 80, True, False, 32, "heads"),
    ([7, 64], [100, 64], 4, 128, 64, False, False, 128, "slots"),
    ([3], [3], 5, 8, 8, False, True, 16, "heads"),
    ([3], [3], 5, 24, 10, False, True, 16, "heads"),      # pairs across lanes, no vectors
    ([9], [70], 2, 72, 38, False, False, 16, "wide"),
    ([9], [70], 2, 40, 6, True, False, 16, "heads"),
    ([17], [30], 33, 32, 0, False, False, 32, "heads"),
    ([17], [30], 3, 104, 0, False, True, 4096, "slots"),
]


def append_check(spec, dtype, bits, k, v, w, eps=EPS, weight=None):
    new, kv, heads, dim, rotary, interleaved, normed, page, layout = spec
    table = A.rotation_table(max(kv), rotary) if rotary else None
    pages, n_pages = page_table(random.Random(1), kv, page)
    caches = [pages_of(layout, n_pages, heads, page, dim, bits, 0x5a) for _ in range(2)]
    plan = A.PagedPlan(new, kv, pages, n_pages=n_pages, page_size=page, q_heads=heads,
                       kv_heads=heads, head_dim=dim)
    mx.taps_mx_append(k, v, *caches, plan, table=table, k_weight=w, eps=eps,
                      interleaved=interleaved)
    left = [[host(t).copy() for t in c] for c in caches]
    at = 0
    for s, (n, m) in enumerate(zip(new, kv)):
        p = np.arange(m - n, m)
        cos, sin = (host(table)[p, i] for i in range(2)) if rotary else (np.zeros((n, 0)),) * 2
        y = M.keys(R.f64(k[at:at + n]), None if w is None else R.f64(w), cos, sin, interleaved, eps)
        for side, x in enumerate((y, R.f64(v[at:at + n]))):
            codes, scales = M.encode(x, bits, dtype)
            place = pages[s, p // page], slice(None), p % page
            for got, want in zip(left[side], (codes, scales)):
                assert np.array_equal(got[place], want), f"sequence {s}, side {side}"
                got[place] = 0x5a
        at += n
    assert all((t == 0x5a).all() for c in left for t in c)   # nothing else was written


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("spec", APPEND)
def test_append(spec, dtype, bits):
    new, kv, heads, dim, normed = spec[0], spec[1], spec[2], spec[3], spec[6]
    say(f"[gpu] mx append {spec} {dtype} {bits}")
    g = gen_of(6)
    # as one projection leaves them; sizes over many binades
    both = torch.randn(sum(new), 2 * heads, dim, generator=g) * \
        torch.exp(2 * torch.randn(sum(new), 2 * heads, dim, generator=g))
    k, v = both.to(dtype).cuda().split(heads, dim=1)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(dtype).cuda() if normed else None
    append_check(spec, dtype, bits, k, v, w)


def test_append_takes_weights_in_32_bits_and_odd_strides():
    g = gen_of(7)
    spec = ([19], [19], 3, 64, 64, False, True, 16, "heads")
    wide = torch.randn(19, 6, 67, generator=g).to(BF16).cuda()
    w = torch.randn(64, generator=g).cuda()
    append_check(spec, BF16, 4, wide[:, :3, 3:], wide[:, 3:, 1:65], w)
    append_check(spec, BF16, 8, wide[:, :3, 2:66], wide[:, 3:, :64], w[:64], eps=0.25)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_append_of_borders(dtype, bits):
    """Elements in the middle of two codes, blocks next to a scale's border, the ends of the
    type's range, zeros of both signs, infinite and NaN elements."""
    largest, least = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    step = torch.finfo(dtype).eps
    rows = []
    for top in (1.0, 6.0, 7.0, 448.0, 464.0, 240.0, 3.5, 2.0 ** -20, 2.0 ** 14, largest,
                largest / 2, largest * 0.75, least, least * 3, 0.0):
        for up in (1.0, 1 - step, 1 + step):
            rows.append([min(top * up, largest), *(top * i / 62 for i in range(31))])
    for scale in (1.0, 2.0 ** -9):   # middles of codes beside the largest
        sizes = M.SIZES[bits]
        middles = (sizes[1:] + sizes[:-1]) / 2
        for at in range(0, len(middles), 15):
            rows.append(([sizes[-1], *middles[at:at + 15]] * 2 + [0.0] * 32)[:32])
            rows[-1] = [x * scale for x in rows[-1]]
    for odd in (math.inf, -math.inf, math.nan):
        rows.append([1.0] * 30 + [odd, -0.0])
    tiny = {BF16: 2.0 ** -133, F16: 2.0 ** -24, F32: 2.0 ** -149}[dtype]
    rows.append([tiny * i for i in range(32)])
    rows.append([-0.0] * 32)
    x = torch.tensor(rows, dtype=torch.float64)
    x = torch.cat([x, -x], dim=1).to(dtype)
    n = len(x)
    k = x.view(n, 1, 64).cuda()
    spec = ([n], [n], 1, 64, 0, False, False, 16, "heads")
    append_check(spec, dtype, bits, k, k.flip(0).contiguous(), None)


def test_append_leaves_what_is_gone():
    """Tokens before a sequence's start are not written; several sequences share pages that are
    only read."""
    caches = [pages_of("heads", 4, 1, 16, 32, 4, 0x5a) for _ in range(2)]
    plan = A.PagedPlan([20, 1], [20, 18], [[-1, 1], [3, 2]], n_pages=4, page_size=16, q_heads=1,
                       kv_heads=1, head_dim=32, kv_starts=[17, 0])
    k = torch.ones(21, 1, 32, dtype=BF16, device="cuda")
    mx.taps_mx_append(k, k, *caches, plan)
    for c in caches:
        for t in c:
            t = host(t)
            written = t[1, 0, 1:4], t[2, 0, 1]
            assert all((x != 0x5a).all() for x in written)
            t[1, 0, 1:4] = t[2, 0, 1] = 0x5a
            assert (t == 0x5a).all()


# ---------------------------------------------------------------------------
# read
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("bits,heads,dim,page,layout", [
    (4, 1, 128, 16, "heads"), (4, 3, 96, 64, "slots"), (4, 5, 40, 32, "wide"),
    (8, 2, 64, 16, "slots"), (8, 3, 80, 128, "wide"), (8, 20, 8, 16, "heads")])
def test_read(bits, heads, dim, page, layout, dtype):
    """Every code with every scale, in the type's range or not, slots asked for twice."""
    say(f"[gpu] mx read {bits} {heads} {dim} {page} {layout} {dtype}")
    rng = np.random.default_rng(3)
    n_pages = 7
    caches = [pages_of(layout, n_pages, heads, page, dim, bits, 0) for _ in range(2)]
    for c in caches:
        for t in c:
            t.copy_(torch.from_numpy(rng.integers(0, 256, t.shape, dtype=np.uint8)))
    n = 201
    slots = rng.integers(0, n_pages * page, n)
    for kind in (torch.int32, torch.int64):
        k, v = mx.taps_mx_read(*caches, torch.from_numpy(slots).to(kind).cuda(), dim, dtype)
        for got, c in zip((k, v), caches):
            place = slots // page, slice(None), slots % page
            want = torch.from_numpy(M.decode(host(c.codes)[place], host(c.scales)[place], dim))
            want = want.to(F32).to(dtype)   # 2^127 x 448 ends 32 bits too
            assert np.array_equal(R.f64(got), R.f64(want), equal_nan=True)


def test_read_refuses_no_slots_and_fills_what_it_is_given():
    caches = [mx.new_pages(3, 2, 16, 64, 4) for _ in range(2)]
    for c in caches:
        c.scales.fill_(127)
        c.codes.fill_(0x22)
    slots = torch.tensor([-1, 0, 47, 48, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    wide = torch.full((6, 5, 70), 7.0, device="cuda")
    k, v = wide[:, 0:2, 3:67], wide[:, 3:5, 2:66]
    got = mx.taps_mx_read(*caches, slots, 64, out=(k, v))
    assert got[0] is k and got[1] is v
    for x in got:
        assert (x[1:3] == 1).all() and x[0].isnan().all() and x[3:].isnan().all()
    far = torch.tensor([2 ** 40, -2 ** 40, 5], device="cuda")
    k, _ = mx.taps_mx_read(*caches, far, 64)
    assert k[:2].isnan().all() and (k[2] == 1).all()
    wide[:, 0:2, 3:67] = 7
    wide[:, 3:5, 2:66] = 7
    assert (wide == 7).all()   # nothing beside them
    none = mx.taps_mx_read(*caches, slots[:0], 64)
    assert none[0].shape == (0, 2, 64)


def test_read_results_stand_apart():
    """One result changes while autograd has the other in use."""
    caches = [mx.new_pages(2, 2, 16, 64, 8) for _ in range(2)]
    k, v = mx.taps_mx_read(*caches, torch.arange(20, device="cuda"), 64, torch.float32)
    w = torch.ones(64, device="cuda", requires_grad=True)
    total = (w * (k + 1)).sum() + (w * k).sum()
    v.fill_(3.0)
    total.backward()
    assert torch.equal(w.grad, torch.full_like(w, 40.0))
    v.mul_(w)
    assert v.requires_grad and not k.requires_grad


def test_append_and_read_back():
    """What is read is what the codes stand for, the nearest to what was appended."""
    g = gen_of(2)
    for bits, dtype in ((4, BF16), (8, BF16), (4, F16), (8, F16), (8, F32)):
        k, v = (randn(g, 50, 3, 72, dtype=dtype) for _ in range(2))
        caches = [mx.new_pages(4, 3, 16, 72, bits) for _ in range(2)]
        plan = A.PagedPlan([50], [50], [[2, 0, 3, 1]], n_pages=4, page_size=16, q_heads=3,
                           kv_heads=3, head_dim=72)
        mx.taps_mx_append(k, v, *caches, plan)
        j = torch.arange(50)
        slots = (torch.tensor([2, 0, 3, 1])[j // 16] * 16 + j % 16).cuda()
        for got, x in zip(mx.taps_mx_read(*caches, slots, 72, dtype), (k, v)):
            codes, scales = M.encode(R.f64(x), bits, dtype)
            assert np.array_equal(R.f64(got), M.decode(codes, scales, 72))


def test_read_of_many_tokens():
    """More than 2^22 workgroups."""
    n = (1 << 22) * 32 + 77
    caches = [mx.new_pages(2, 1, 16, 8, 4) for _ in range(2)]
    for c in caches:
        c.scales.fill_(127)
        c.codes.copy_(torch.arange(32, dtype=torch.uint8, device="cuda").view(2, 1, 16, 1))
    slots = torch.arange(n, dtype=torch.int32, device="cuda") % 32
    k, v = mx.taps_mx_read(*caches, slots, 8)
    want = torch.from_numpy(M.SIZES[4]).to(BF16).cuda()[torch.arange(32, device="cuda") % 8]
    want = torch.where(torch.arange(32, device="cuda") % 16 >= 8, -want, want)
    for x in (k, v):
        for a in range(0, n, 1 << 24):
            assert torch.equal(x[a:a + (1 << 24), 0, 0], want[slots[a:a + (1 << 24)].long()])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def attend_case(spec, dtype, bits, layout="heads", seed=4):
    """(q, caches, plan, keys and values in 64 bits per sequence, page table); slots that hold no
    key, or one before the sequence's start, have codes and scales that are NaN."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    g = gen_of(seed)
    starts = options.get("kv_starts", [0] * len(kv_lens))
    pages, n_pages = page_table(random.Random(seed), kv_lens, page)
    caches = [pages_of(layout, n_pages, kv_heads, page, dim, bits, 255) for _ in range(2)]
    kept = []
    for s, n in enumerate(kv_lens):
        both = []
        for c in caches:
            x = np.full((n, kv_heads, dim), math.nan)
            x[starts[s]:] = set_keys(c, pages, s, R.f64(torch.randn(
                n - starts[s], kv_heads, dim, generator=g)), page, starts[s])
            both.append(x)
        kept.append(tuple(both))
        pages[s, :starts[s] // page] = -1
    q = randn(g, sum(q_lens), q_heads, dim, dtype=dtype, scale=1.5)
    plan = A.PagedPlan(q_lens, kv_lens, pages, n_pages=n_pages, page_size=page, q_heads=q_heads,
                       kv_heads=kv_heads, head_dim=dim, **options)
    return q, caches, plan, kept, pages


MORE = [
    ([1], [1], 1, 1, 8, 16, {}),
    ([1], [31], 4, 4, 24, 16, {}),
    ([3], [50], 4, 2, 32, 16, {}),
    ([1, 1], [640, 1300], 16, 1, 128, 64, {}),           # 16 rows, and 17 and more
    ([1, 1], [640, 1300], 17, 1, 128, 64, {}),
    ([4, 4, 3], [640, 1300, 3], 8, 2, 96, 32, {}),
    ([5, 1], [640, 1300], 8, 2, 64, 32, {"units": 4096}),
    ([4], [9000], 4, 1, 128, 64, {"units": 4096, "window": 5000}),
    ([2, 2], [700, 30], 8, 2, 104, 16, {"kv_starts": [300, 29]}),
    # more items than units: of 128 rows, of 17 to 32 and of up to 16
    ([40] * 11 + [10] * 12 + [3] * 12, [40] * 11 + [150, 11, 32, 31] * 6, 16, 8, 128, 16, {}),
    ([40] * 11 + [10] * 12 + [3] * 12, [90] * 11 + [150, 11, 32, 31] * 6, 16, 8, 64, 32,
     {"window": 30}),
    ([40] * 11 + [9] * 12 + [3] * 12, [70] * 11 + [150, 11, 32, 31] * 6, 16, 8, 96, 64,
     {"kv_starts": [33] * 11 + [7] * 24}),
    ([1] * 30 + [4] * 5, [5, 700, 64, 65, 33] * 7, 32, 8, 128, 16, {}),
    ([1] * 30 + [4] * 5, [5, 700, 64, 65, 33] * 7, 32, 8, 72, 64, {"window": 50}),
]


@pytest.mark.parametrize("spec,dtype,bits", [
    *((spec, *kind) for spec in ATTEND + WIDE for kind in ((BF16, 4), (F16, 8))),
    *((spec, dtype, bits) for spec in MORE for dtype in (BF16, F16) for bits in (4, 8))])
def test_attend(spec, dtype, bits):
    say(f"[gpu] mx attend {spec} {dtype} {bits}")
    q, caches, plan, kept, _ = attend_case(spec, dtype, bits)
    assert wide_items(plan) or spec not in WIDE
    out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
    torch.cuda.synchronize()
    attend_check(spec, q, kept, out, lse, spec[4] ** -0.5, dtype)
    assert torch.equal(mx.taps_mx_attend(q, *caches, plan), out)   # without lse, and again


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("layout", ["slots", "wide"])
def test_attend_layouts(layout, bits):
    """Caches in other orders, queries and outputs that are slices, a scale of one's own."""
    spec = ([40, 1, 130], [300, 90, 130], 6, 2, 96, 32, {})
    say(f"[gpu] mx attend layout {layout} {bits}")
    q, caches, plan, kept, _ = attend_case(spec, F16, bits, layout)
    wide_q = torch.full((q.shape[0], 9, 104), math.nan, dtype=F16, device="cuda")
    wide_out = torch.full((8, q.shape[0], 96), 3.0, dtype=F16, device="cuda")
    wide_q[:, 2:8, 8:] = q
    out = wide_out[1:7].transpose(0, 1)
    got = mx.taps_mx_attend(wide_q[:, 2:8, 8:], *caches, plan, scale=0.31, out=out)
    assert got is out
    attend_check(spec, q, kept, out, None, 0.31, F16)
    assert (wide_out[0] == 3).all() and (wide_out[7] == 3).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_attend_large_scores(bits):
    """Scores in the hundreds: one key takes all, maxima rise late and in steps."""
    spec = ([130, 1, 3], [600, 2000, 900], 4, 2, 64, 16, {"units": 1024})
    for dtype in (BF16, F16):
        q, caches, plan, kept, pages = attend_case(spec, dtype, bits)
        q = (q * 30).contiguous()
        out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
        attend_check(spec, q, kept, out, lse, 0.125, dtype)
        rising = [(set_keys(caches[0], pages, s, k * np.linspace(0.02, 1, len(k))[:, None, None],
                            16), v) for s, (k, v) in enumerate(kept)]
        out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
        attend_check(spec, q, rising, out, lse, 0.125, dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_attend_many_small_numerators(dtype, bits):
    """One key above thousands whose numerators lie below the smallest normal 16-bit numbers, and
    together weigh as much as it does; the key comes first, last or between."""
    n, dim, page = 9000, 64, 64
    g = gen_of(8)
    for q_len, at in ((1, 0), (1, n - 1), (3, 77), (40, 4000)):
        pages, n_pages = page_table(random.Random(2), [n], page)
        caches = [pages_of("heads", n_pages, 1, page, dim, bits, 255) for _ in range(2)]
        k = np.zeros((n, 1, dim))
        k[:, 0, 0] = -12.0 + 2.0 * host(torch.randint(0, 2, (n,), generator=g))
        k[at, 0, 0] = 0
        q = torch.zeros(q_len, 1, dim, dtype=dtype)
        q[:, 0, 0] = 8.0
        kept = [(set_keys(caches[0], pages, 0, k, page),
                 set_keys(caches[1], pages, 0, R.f64(torch.randn(n, 1, dim, generator=g)), page))]
        spec = ([q_len], [n], 1, 1, dim, page, {})
        plan = A.PagedPlan([q_len], [n], pages, n_pages=n_pages, page_size=page, q_heads=1,
                           kv_heads=1, head_dim=dim)
        out, lse = mx.taps_mx_attend(q.cuda(), *caches, plan, lse=True)
        attend_check(spec, q, kept, out, lse, 0.125, dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", [
    ([4, 30], [4, 200], 4, 2, 128, 16, {}),                  # few rows, several tokens
    ([4, 2], [300, 77], 2, 1, 64, 16, {"window": 20}),
    ([70, 3], [70, 90], 2, 2, 64, 16, {"window": 20}),
    ([140], [500], 2, 1, 96, 32, {"window": 65}),
    ([300], [330], 4, 2, 128, 64, {"units": 1}),
    ([40], [1500], 8, 2, 128, 64, {"units": 4096}),
    ([3], [1500], 4, 2, 96, 64, {"units": 4096}),
    ([300], [1700], 4, 2, 128, 64, {"units": 1}),            # 256 rows an item
    ([300], [2900], 4, 2, 80, 16, {"units": 1, "window": 1500}),
    # more items than units
    ([40] * 12 + [10] * 12 + [3] * 12, [60] * 12 + [150, 11, 32, 31] * 6, 16, 8, 128, 16, {}),
    ([3] * 40, [60, 70, 150, 11, 32] * 8, 8, 8, 64, 16, {"window": 25}),
])
def test_attend_blocks_of_nan(spec, dtype, bits):
    """Blocks that are NaN, among the new tokens and before: they reach the tokens that see them
    and no others."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    say(f"[gpu] mx attend nan {spec} {dtype} {bits}")
    q, caches, plan, kept, pages = attend_case(spec, dtype, bits)
    rng = random.Random(5)
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for which in (1, 1, 0):
            j = m - 1 - rng.randrange(min(m, n + 40))   # a new token, or one just before them
            h, b = rng.randrange(kv_heads), rng.randrange(-(-dim // 32))
            caches[which].scales[pages[s, j // page], h, j % page, b] = 255
            kept[s][which][j, h, 32 * b:32 * b + 32] = math.nan
    out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
    want_bad = clean = at = 0
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        with np.errstate(invalid="ignore"):
            want, bound, _, _ = R.attend(R.f64(q[at:at + n]), *kept[s], m - n, 0, True,
                                         options.get("window", 0), dim ** -0.5, dtype)
        got = R.f64(out[at:at + n])
        bad = np.isnan(want)
        assert np.array_equal(bad, np.isnan(got)), "not the same outputs are NaN"
        R.check(np.where(bad, 0, got), np.where(bad, 0, want), np.where(bad, 1, bound), "finite")
        want_bad, clean = want_bad + bad.sum(), clean + (~bad).sum()
        at += n
    # with one key head and a window, all tokens see the key that is NaN
    assert want_bad and (clean or kv_heads == 1)


NOT_FINITE = [
    ([4, 30], [4, 200], 4, 2, 128, 16, {}),                  # few rows, several tokens
    ([4, 2], [300, 77], 2, 1, 64, 16, {"window": 20}),
    ([9], [1500], 8, 2, 96, 64, {"units": 4096}),            # 17 to 32 rows, in pieces
    ([140], [500], 2, 1, 96, 32, {"window": 65}),
    ([300], [330], 4, 2, 128, 64, {"units": 1}),
    ([40], [1500], 8, 2, 128, 64, {"units": 4096}),
    ([300], [1700], 4, 2, 128, 64, {"units": 1}),            # 256 rows an item
    # more items than units
    ([40] * 12 + [10] * 12 + [3] * 12, [60] * 12 + [150, 11, 32, 31] * 6, 16, 8, 64, 16, {}),
    ([3] * 40, [60, 70, 150, 11, 32] * 8, 8, 8, 64, 16, {"window": 25}),
]


def not_finite_check(spec, q, kept, out, lse, dtype):
    """The outputs and sums that are not finite are those that cannot be, the others near."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    bad, total = np.zeros(2, dtype=int), np.zeros(2, dtype=int)
    at = 0
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        with np.errstate(invalid="ignore"):
            *of_out, w_lse, b_lse = R.attend(R.f64(q[at:at + n]), *kept[s], m - n, 0, True,
                                             options.get("window", 0), dim ** -0.5, dtype)
        for i, (x, want, bound) in enumerate(((out, *of_out), (lse, w_lse, b_lse))):
            got, off = R.f64(x[at:at + n]), ~np.isfinite(want)
            assert np.array_equal(off, ~np.isfinite(got)), "not the same ones are finite"
            assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
            # a bound of infinity (scores of -inf) times 0 is that of a sum of zeros: 0
            bound = np.where(np.isnan(bound), 0, bound)
            R.check(np.where(off, 0, got), np.where(off, 0, want), np.where(off, 1, bound),
                    ("out", "lse")[i])
            bad[i], total[i] = bad[i] + off.sum(), total[i] + off.size
        at += n
    return bad, total


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", NOT_FINITE)
def test_attend_lse_beside_blocks_of_nan(spec, dtype, bits):
    """A row's sum of exponentials has nothing to do with the values, and is NaN where a key is."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    say(f"[gpu] mx attend nan lse {spec} {dtype} {bits}")
    for which in (1, 0):
        q, caches, plan, kept, pages = attend_case(spec, dtype, bits)
        rng = random.Random(7)
        for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
            j = m - 1 - rng.randrange(min(m, n + 16))   # a new token, or one just before them
            h, b = rng.randrange(kv_heads), rng.randrange(-(-dim // 32))
            caches[which].scales[pages[s, j // page], h, j % page, b] = 255
            kept[s][which][j, h, 32 * b:32 * b + 32] = math.nan
        out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
        bad, total = not_finite_check(spec, q, kept, out, lse, dtype)
        assert 0 < bad[0] and (bad[0] < total[0] or kv_heads == 1)
        assert bad[1] == 0 if which else dim * bad[1] == bad[0]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("spec", NOT_FINITE)
def test_attend_beyond_the_range_of_fp16(spec, bits):
    """Blocks of values, and single elements of keys, that are infinite in fp16: they reach the
    tokens that see them and no others."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    say(f"[gpu] mx attend infinities {spec} {bits}")
    q, caches, plan, kept, pages = attend_case(spec, F16, bits)
    rng = random.Random(9)
    for s, (n, m) in enumerate(zip(q_lens, kv_lens)):
        for which in (1, 1, 0):
            j = m - 1 - rng.randrange(min(m, n + 16))
            h, b = rng.randrange(kv_heads), rng.randrange(dim // 32)
            place = pages[s, j // page], h, j % page
            codes = caches[which].codes[place][4 * bits * b:4 * bits * (b + 1)]
            if which:   # 2^40 times what they stood for, 2^-17 or more
                caches[which].scales[place][b] += 40
                x = kept[s][1][j, h, 32 * b:32 * b + 32]
                kept[s][1][j, h, 32 * b:32 * b + 32] = np.where(
                    x == 0, 0, np.copysign(math.inf, x))
            else:       # one element, 2^0 x 2^30, among zeros
                codes.zero_()
                codes[0] = 2 if bits == 4 else 0x38
                caches[which].scales[place][b] = 157
                kept[s][0][j, h, 32 * b:32 * b + 32] = [math.inf] + [0] * 31
    # (scores of a row lie within a few units of each other: no numerator rounds to nothing)
    out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
    bad, total = not_finite_check(spec, q, kept, out, lse, F16)
    assert 0 < bad[0] and (bad[0] < total[0] or kv_heads == 1)


@pytest.mark.parametrize("dim", [64, 96, 128])
def test_tokens_without_keys(dim):
    """Sequences that have lost all their keys: zeros, whatever earlier workgroups left in LDS."""
    n, kv = 300, 20
    nans = [pages_of("heads", 8, 1, 16, dim, 4, 255) for _ in range(2)]
    for heads in (1, 64):
        plan = A.PagedPlan([1] * n, [kv] * n, np.full((n, 2), -1), n_pages=8, page_size=16,
                           q_heads=heads, kv_heads=1, head_dim=dim, kv_starts=[kv] * n)
        spoil = A.PagedPlan([96], [128], np.arange(8)[None], n_pages=8, page_size=16, q_heads=1024,
                            kv_heads=1, head_dim=dim, causal=False)
        q, sq = randn(gen_of(1), n, heads, dim), randn(gen_of(2), 96, 1024, dim)
        assert mx.taps_mx_attend(sq, *nans, spoil).isnan().all()
        out, lse = mx.taps_mx_attend(q, *nans, plan, lse=True)
        assert (out == 0).all() and (lse == -math.inf).all()


def test_attend_far_offsets():
    """Caches of more than 2^32 bytes, a sequence at their far end; append and read there too."""
    page, heads, dim, n_pages = 64, 8, 128, 140000   # 4.6e9 bytes of codes each
    g = gen_of(1)
    caches = [mx.MxPages(torch.empty((n_pages, heads, page, 64), dtype=torch.uint8, device="cuda"),
                         torch.empty((n_pages, heads, page, 4), dtype=torch.uint8, device="cuda"))
              for _ in range(2)]
    kv = [200, 150]
    pages = np.array([[139999, 3, 139997, 132769], [139990, 139991, 5, -1]], dtype=np.int32)
    kept = [tuple(set_keys(c, pages, s, R.f64(torch.randn(n, heads, dim, generator=g)), page)
                  for c in caches) for s, n in enumerate(kv)]
    plan = A.PagedPlan([1, 40], kv, pages, n_pages=n_pages, page_size=page, q_heads=8, kv_heads=8,
                       head_dim=128)
    q = randn(g, 41, 8, 128)
    out = mx.taps_mx_attend(q, *caches, plan)
    attend_check(([1, 40], kv, 8, 8, 128, page, {}), q, kept, out, None, 128 ** -0.5, BF16)
    k, v = randn(g, 41, 8, 128), randn(g, 41, 8, 128)
    mx.taps_mx_append(k, v, *caches, plan)
    slots = torch.tensor([132769 * 64 + 7, 5 * 64 + 21], device="cuda")
    for kind in (torch.int32, torch.int64):
        for got, x in zip(mx.taps_mx_read(*caches, slots.to(kind), 128), (k, v)):
            codes, scales = M.encode(R.f64(x[[0, 40]]), 4, BF16)
            assert np.array_equal(R.f64(got), M.decode(codes, scales, 128))


@pytest.mark.parametrize("bits,spec", [
    (4, ([3, 10, 40, 1], [300, 200, 90, 17], 4, 2, 128, 16, {})),
    (8, ([3, 10, 40, 1], [300, 200, 90, 17], 4, 2, 64, 32, {"window": 150})),
    (8, ([300], [1700], 4, 2, 96, 16, {"units": 1})),        # 256 rows an item
])
def test_slots_far_apart(bits, spec):
    """Slots as far apart as they may be, pages and heads between them; both kinds of strides odd
    in all but what is asked for."""
    q_lens, kv_lens, q_heads, kv_heads, dim, page, options = spec
    say(f"[gpu] mx far slots {bits} {spec}")
    q, caches, plan, _, pages = attend_case(spec, BF16, bits)
    far = []
    for c in caches:
        apart = [2 ** 27 - 16, 2 ** 27 - 1]
        far.append(mx.MxPages(*(torch.empty_strided(
            t.shape, (kv_heads * size, size, slot, 1), dtype=torch.uint8, device="cuda").copy_(t)
            for t, slot, size in zip(c, apart, (c.codes.shape[3] + 16, c.scales.shape[3] + 3)))))
    want, want_lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
    got, lse = mx.taps_mx_attend(q, *far, plan, lse=True)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    k, v = (randn(gen_of(5), sum(q_lens), kv_heads, dim) for _ in range(2))
    every = torch.arange(caches[0].codes.shape[0] * page, device="cuda")
    for c in (caches, far):
        mx.taps_mx_append(k, v, *c, plan, table=A.rotation_table(max(kv_lens), dim))
    for a, b in zip(caches, far):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    for a, b in zip(*(mx.taps_mx_read(*c, every, dim) for c in (caches, far))):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))   # NaN where nothing is
    del far
    torch.cuda.empty_cache()


def test_pages_that_sequences_share():
    """Two sequences whose first pages are the same ones, only read."""
    spec = ([1, 3], [200, 180], 8, 2, 128, 16, {})
    q, caches, _, kept, pages = attend_case(spec, BF16, 4)
    pages[1, :5] = pages[0, :5]
    kept[1] = tuple(np.concatenate([a[:80], b[80:]]) for a, b in zip(*kept))
    plan = A.PagedPlan(*spec[:2], pages, n_pages=caches[0].codes.shape[0], page_size=16, q_heads=8,
                       kv_heads=2, head_dim=128)
    out, lse = mx.taps_mx_attend(q, *caches, plan, lse=True)
    attend_check(spec, q, kept, out, lse, 128 ** -0.5, BF16)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

KV = [70, 1, 333, 128]


def _step(bits, dtype=BF16):
    """A decoding step's tensors: q, k, v, weights, table, positions, caches, plan, new slots."""
    g = gen_of(12)
    pages, n_pages = page_table(random.Random(3), KV, 16)
    caches = [mx.new_pages(n_pages, 2, 16, 64, bits) for _ in range(2)]
    for s, n in enumerate(KV):
        for c in caches:
            set_keys(c, pages, s, R.f64(torch.randn(n, 2, 64, generator=g)), 16)
    plan = A.PagedPlan([1] * 4, KV, pages, n_pages=n_pages, page_size=16, q_heads=8, kv_heads=2,
                       head_dim=64)
    qkv = randn(g, 4, 12, 64, dtype=dtype, scale=2)
    w = randn(g, 64, dtype=dtype)
    table = A.rotation_table(400, 64)
    positions = torch.tensor(KV, dtype=torch.int32).cuda() - 1
    slots = torch.tensor([pages[s, (n - 1) // 16] * 16 + (n - 1) % 16 for s, n in enumerate(KV)],
                         dtype=torch.int32).cuda()
    return qkv, w, table, positions, caches, plan, slots


def _run_step(qkv, w, table, positions, caches, plan, slots, **kw):
    q, k, v = qkv.split((8, 2, 2), dim=1)
    q, _ = A.taps_norm_rotate(q, None, w, None, table, positions=positions, **kw)
    mx.taps_mx_append(k, v, *caches, plan, table=table, k_weight=w, **kw)
    back = mx.taps_mx_read(*caches, slots, 64, **kw)
    return mx.taps_mx_attend(q, *caches, plan, **kw), *back


@pytest.mark.parametrize("bits", [4, 8])
def test_step_agrees_with_attention_over_16_bits(bits):
    """Over a 16-bit cache of what the codes stand for, attention gives the same within roundings
    of its numerators and results, and the new tokens are among the keys."""
    step = _step(bits)
    qkv, w, table, positions, caches, plan, slots = step
    out, k, v = _run_step(*step)
    n_pages = caches[0].codes.shape[0]
    every = torch.arange(n_pages * 16, dtype=torch.int32, device="cuda")
    half = [x.view(n_pages, 16, 2, 64).transpose(1, 2).contiguous()
            for x in mx.taps_mx_read(*caches, every, 64)]
    for c, x in zip(half, (k, v)):
        assert torch.equal(c[slots.long() // 16, :, slots.long() % 16], x)
    q, _ = A.taps_norm_rotate(qkv[:, :8], None, w, None, table, positions=positions)
    want, lse = A.taps_attend(q, *half, plan, lse=True)
    got, mine = mx.taps_mx_attend(q, *caches, plan, lse=True)
    assert torch.equal(got, out)
    # both round numerators and results by 2^-8 of at most the largest value
    most = half[1].abs().max().item()
    assert (got.float() - want.float()).abs().max().item() <= 4 * 2.0 ** -8 * most
    # sums of 64 products and of up to 333 numerators, each within 2^-24 of the scores' size
    size = (q.float().abs().max() * half[0].float().abs().max() * 64 * 0.125).item()
    assert (mine - lse).abs().max().item() <= (4 * 64 + 2 * 333) * 2.0 ** -24 * (size + 1)


@pytest.mark.parametrize("bits", [4, 8])
def test_step_in_a_graph(bits):
    """Captured once, replayed with other inputs between eager work."""
    step = _step(bits)
    qkv = step[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run_step(*step)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _run_step(*step)
    g = gen_of(30)
    for _ in range(4):
        qkv.copy_(randn(g, *qkv.shape, scale=2))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        want = _run_step(*step)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("spec", [
    ([1, 4], [9000, 700], 8, 2, 128, 64, {"units": 256}),        # few rows
    ([10, 40], [9000, 700], 8, 2, 64, 16, {"units": 4096}),
    ([300], [2900], 4, 2, 128, 64, {"units": 64}),               # 256 rows an item
])
def test_pieces_in_a_graph(spec):
    """Attention whose keys are split, its workspace the graph's, between eager work."""
    say(f"[gpu] mx pieces in a graph {spec}")
    q, caches, plan, _, _ = attend_case(spec, BF16, 8)
    assert plan.workspace_bytes
    want = mx.taps_mx_attend(q, *caches, plan, lse=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mx.taps_mx_attend(q, *caches, plan, lse=True)
    g = gen_of(31)
    for _ in range(4):
        graph.replay()
        torch.full((1 << 22,), math.nan, device="cuda")
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        q.copy_(randn(g, *q.shape, scale=1.5))
        want = mx.taps_mx_attend(q, *caches, plan, lse=True)


def test_step_on_another_stream():
    """The stream argument, while the current stream is busy with other memory."""
    step = _step(4)
    want = _run_step(*step)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        noise = [torch.full((1 << 20,), math.nan, device="cuda") for _ in range(4)]
        side.wait_stream(torch.cuda.current_stream())
        got = _run_step(*step, stream=side)
        del noise
        torch.full((1 << 20,), math.nan, device="cuda")
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gradients_raise():
    qkv, w, table, positions, caches, plan, slots = _step(8)
    q = qkv[:, :8].clone().requires_grad_()
    with pytest.raises(RuntimeError, match="taps_mx_attend has no gradient"):
        mx.taps_mx_attend(q, *caches, plan).sum().backward()
    with torch.no_grad():
        assert not mx.taps_mx_attend(q, *caches, plan).requires_grad


def test_tangents_raise():
    """Forward mode, over either cache: queries, weights and a cache with tangents."""
    qkv, w, table, positions, caches, plan, _ = _step(4)
    q = qkv[:, :8].contiguous()
    half = [torch.zeros(caches[0].codes.shape[0], 2, 16, 64, dtype=BF16, device="cuda")
            for _ in range(2)]

    def norm(q, w):
        return A.taps_norm_rotate(q, None, w, None, table, positions=positions)

    def attend(q, k):
        return A.taps_attend(q, k, half[1], plan)

    def mx_attend(q):
        return mx.taps_mx_attend(q, *caches, plan)
    for call, args in ((norm, (q, w)), (attend, (q, half[0])), (mx_attend, (q,))):
        with torch.autograd.forward_ad.dual_level():
            call(*args)
            for i, x in enumerate(args):
                dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
                with pytest.raises(RuntimeError, match="has no gradient"):
                    call(*args[:i], dual, *args[i + 1:])
        call(*args)


def test_gpu_refusals():
    q = torch.zeros(4, 8, 64, dtype=BF16, device="cuda")
    c = mx.new_pages(2, 8, 16, 64, 4)
    table = A.rotation_table(16, 64)
    shape = {"n_pages": 2, "page_size": 16, "q_heads": 8, "kv_heads": 8}
    plan = A.PagedPlan([4], [20], [[0, 1]], head_dim=64, **shape)
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(TapsError, match="positions up to 20"):
        mx.taps_mx_append(q, q, c, c, plan, table=table)
    with pytest.raises(ValueError, match="k_cache is MxPages.1 pages"):
        mx.taps_mx_append(q, q, mx.MxPages(c.codes[:1], c.scales[:1]), c, plan)
    with pytest.raises(ValueError, match="v_cache is MxPages.* 4 blocks"):
        mx.taps_mx_append(q, q, c, mx.new_pages(2, 8, 16, 128, 4), plan)
    with pytest.raises(ValueError, match="keys of 4 bits beside values of 8"):
        mx.taps_mx_attend(q, c, mx.new_pages(2, 8, 16, 64, 8), plan)
    with pytest.raises(ValueError, match="not on the GPU"):
        mx.taps_mx_attend(q, mx.MxPages(c.codes.cpu(), c.scales.cpu()), c, plan)
    with pytest.raises(ValueError, match="is torch.float16"):
        mx.taps_mx_append(q, q.half(), c, c, plan)
    with pytest.raises(ValueError, match="not supported"):
        mx.taps_mx_append(q.double(), q.double(), c, c, plan)
    with pytest.raises(TapsError, match="neither TAPS_BF16"):
        mx.taps_mx_attend(q.float(), c, c, plan)
    with pytest.raises(TapsError, match="scale"):
        mx.taps_mx_attend(q, c, c, plan, scale=0.0)
    with pytest.raises(ValueError, match="q is"):
        mx.taps_mx_attend(q[:3], c, c, plan)
    short = A.PagedPlan([4], [3], [[0]], head_dim=64, **shape)
    with pytest.raises(TapsError, match="more new tokens than keys"):
        mx.taps_mx_append(q, q, c, c, short)
    odd = A.PagedPlan([4], [20], [[0, 1]], head_dim=60, **shape)
    with pytest.raises(TapsError, match="multiple of 8"):
        mx.taps_mx_append(q[..., :60], q[..., :60], c, c, odd)
    unaligned = torch.zeros(2 * 8 * 16 * 32 + 8, dtype=torch.uint8, device="cuda")[8:]
    with pytest.raises(TapsError, match="multiples of 16 bytes"):
        mx.taps_mx_append(q, q, mx.MxPages(unaligned.view(2, 8, 16, 32), c.scales), c, plan)
    with pytest.raises(ValueError, match="slots"):
        mx.taps_mx_read(c, c, slots.float(), 64)
    with pytest.raises(ValueError, match="slots"):
        mx.taps_mx_read(c, c, slots.view(1, 3), 64)
    with pytest.raises(ValueError, match="not on the GPU"):
        mx.taps_mx_read(c, c, slots.cpu(), 64)
    with pytest.raises(ValueError, match="4 blocks"):
        mx.taps_mx_read(c, c, slots, 128)
    with pytest.raises(TapsError, match="multiple of 8"):
        mx.taps_mx_read(c, c, slots, 60)
    with pytest.raises(ValueError, match="not supported"):
        mx.taps_mx_read(c, c, slots, 64, dtype=torch.float64)
    with pytest.raises(TapsError, match="power of two"):
        d = mx.new_pages(2, 8, 24, 64, 4)
        mx.taps_mx_read(d, d, slots, 64)
    with pytest.raises(ValueError, match="k is"):
        mx.taps_mx_read(c, c, slots, 64, out=(q, q))
