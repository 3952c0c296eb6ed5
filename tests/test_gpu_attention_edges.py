"""The attention operators on the GPU where they meet the edges of what they take: items
without keys, values that are infinite or NaN beside finite ones, weights far below a
row's largest, gradients of gradients."""
import math

import numpy as np
import pytest
import torch

import attention_reference as R
from paper_2301_04285_amd import attention as A

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def say(*a):
    print(*a, flush=True)


def gen_of(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(gen, *shape, dtype=BF16, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()


def paged(x, page):
    """x [keys, heads, dim] as a cache [pages, heads, page, dim], NaN where x has no key."""
    n, heads, dim = x.shape
    pages = max(1, -(-n // page))
    c = torch.full((pages * page, heads, dim), math.nan, dtype=x.dtype)
    c[:n] = x
    return c.view(pages, page, heads, dim).transpose(1, 2).contiguous().cuda()


# ---------------------------------------------------------------------------
# items without keys
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_tokens_without_keys_and_many_heads(dim, causal):
    """One token of 64 query heads to a key head whose sequence has lost all its keys: zeros,
    whatever earlier workgroups left in LDS."""
    n, kv = 700, 20
    say(f"[gpu] attend no keys {dim} {causal}")
    nans = torch.full((8, 1, 16, dim), math.nan, dtype=BF16, device="cuda")
    plan = A.PagedPlan([1] * n, [kv] * n, np.full((n, 2), -1), n_pages=8, page_size=16, q_heads=64,
                       kv_heads=1, head_dim=dim, kv_starts=[kv] * n, causal=causal)
    q = randn(gen_of(1), n, 64, dim)
    # one sequence whose keys and values are all NaN, enough rows to visit every compute unit
    rows = 96
    pages = np.arange(8)[None]
    spoil = A.PagedPlan([rows], [128], pages, n_pages=8, page_size=16, q_heads=1024, kv_heads=1,
                        head_dim=dim, causal=False)
    sq = randn(gen_of(2), rows, 1024, dim)
    for _ in range(3):
        assert A.taps_attend(sq, nans, nans, spoil).isnan().all()
        out, lse = A.taps_attend(q, nans, nans, plan, lse=True)
        assert (out == 0).all() and (lse == -math.inf).all()


# ---------------------------------------------------------------------------
# elements that are not rotated
# ---------------------------------------------------------------------------

def same_specials(got, want, bound, what):
    """Infinite and NaN where the definition is, finite elsewhere and within the bound."""
    got = R.f64(got)
    odd = ~np.isfinite(want)
    assert np.array_equal(np.where(odd, got, 0), np.where(odd, want, 0), equal_nan=True), what
    R.check(np.where(odd, 0, got), np.where(odd, 0, want), np.where(odd, 0, bound), what)


PARTS = [   # dim, rotary, interleaved: by fours of elements, and element by element
    (128, 64, False), (128, 64, True), (96, 48, True), (64, 0, False), (8, 0, False),
    (36, 18, False), (37, 10, True), (101, 50, False), (7, 0, False), (256, 2, True),
]


def with_specials(x, rotary):
    """Every unrotated element in turn, and sign, has an infinity or a NaN in some row."""
    dim = x.shape[-1]
    rows = x.view(-1, dim)
    values = (math.inf, -math.inf, math.nan)
    for r in range(min(len(rows), dim - rotary)):
        rows[r, rotary + (r * 5 + 1) % (dim - rotary)] = values[r % 3]
    return x


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("spec", PARTS)
def test_unrotated_elements_stay(spec, dtype):
    """An infinite or NaN element that is not rotated reaches no other element of its head,
    forwards, backwards and on the way to a cache; without a rotation and a norm keys are
    copied."""
    dim, rotary, interleaved = spec
    say(f"[gpu] unrotated {spec} {dtype}")
    tokens, heads = 40, 3
    g = gen_of(21)
    x = with_specials(randn(g, 1, tokens, heads, dim, dtype=dtype), rotary)
    table = A.rotation_table(tokens, rotary) if rotary else None
    cos, sin = np.zeros((1, tokens, 0)), np.zeros((1, tokens, 0))
    if rotary:
        cos, sin = (R.f64(table)[None, :, i] for i in range(2))
    y, bound = R.norm_rotate(R.f64(x), None, cos, sin, interleaved, 1e-6, dtype)
    out, _ = A.taps_norm_rotate(x, None, None, None, table, interleaved=interleaved)
    same_specials(out, y, bound, "output")
    dx, b, _, _ = R.norm_rotate_gradients(R.f64(x), R.f64(x), None, cos, sin, interleaved, 1e-6,
                                          dtype, None)
    grads = A.taps_norm_rotate_backward(x, None, x, None, None, None, table,
                                        interleaved=interleaved)
    same_specials(grads[0], dx, b, "gradient")
    page = 16
    caches = [torch.zeros(3, heads, page, dim, dtype=dtype, device="cuda") for _ in range(2)]
    plan = A.PagedPlan([tokens], [tokens], [[2, 0, 1]], n_pages=3, page_size=page, q_heads=heads,
                       kv_heads=heads, head_dim=dim)
    A.taps_cache_append(x[0], x[0], *caches, plan, table=table, interleaved=interleaved)
    left = [c[[2, 0, 1]].transpose(1, 2).flatten(0, 1)[:tokens] for c in caches]
    same_specials(left[0], y[0], bound[0], "key")
    assert np.array_equal(R.f64(left[1]), R.f64(x[0]), equal_nan=True)
    if not rotary:
        assert np.array_equal(R.f64(left[0]), R.f64(x[0]), equal_nan=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("spec", PARTS[:3] + PARTS[5:8])
def test_unrotated_elements_stay_with_a_norm(spec, dtype):
    """The norm of a row with an infinity is infinite: that element becomes NaN and its
    neighbours 0.  An infinite gradient reaches its own element's weight gradient alone."""
    dim, rotary, interleaved = spec
    say(f"[gpu] unrotated, normed {spec} {dtype}")
    g = gen_of(22)
    x = randn(g, 1, 5, 2, dim, dtype=dtype)
    grad = randn(g, 1, 5, 2, dim, dtype=dtype)
    w = (1 + 0.3 * torch.randn(dim, generator=g)).to(dtype).cuda()
    table = A.rotation_table(5, rotary)
    cos, sin = (R.f64(table)[None, :, i] for i in range(2))
    bad = x.clone()
    bad[0, 2, 1, rotary + 1] = math.inf
    with np.errstate(invalid="ignore"):
        y, bound = R.norm_rotate(R.f64(bad), R.f64(w), cos, sin, interleaved, 1e-6, dtype)
    out, _ = A.taps_norm_rotate(bad, None, w, None, table, interleaved=interleaved)
    same_specials(out, y, np.nan_to_num(bound), "output")
    grad[0, 3, 0, rotary + 2] = -math.inf
    grad[0, 4, 1, dim - 1] = math.inf
    with np.errstate(invalid="ignore"):
        _, _, dw, bw = R.norm_rotate_gradients(R.f64(grad), R.f64(x), R.f64(w), cos, sin,
                                               interleaved, 1e-6, dtype, dtype)
    got = A.taps_norm_rotate_backward(grad, None, x, None, w, None, table,
                                      interleaved=interleaved)[2]
    assert np.isinf(dw).sum() == 2
    same_specials(got, dw, bw, "weight gradient")


# ---------------------------------------------------------------------------
# weights far below a row's largest
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", [
    # tokens, keys, dim, where the largest weight is
    (1, 1500, 64, 0), (1, 1500, 128, 1499), (3, 1500, 96, 700), (40, 1500, 64, 0),
    (40, 1500, 128, 300), (300, 2300, 128, 0),   # the last in strips of 256 rows
])
def test_weights_far_below_the_largest(spec, dtype):
    """One key whose value is 0 above thousands that lie e^-17 to e^-20 below: the result is
    theirs.  Numerators of 16 bits reach 35 binary places below the largest."""
    new, n, dim, at = spec
    say(f"[gpu] attend far below {spec} {dtype}")
    g = gen_of(31)
    k = torch.zeros(n, 1, dim, dtype=dtype)
    k[:, 0, 0] = -17 - 0.25 * torch.randint(0, 13, (n,), generator=g).to(dtype)
    v = (1 + 0.25 * torch.randn(n, 1, dim, generator=g)).to(dtype)
    k[at], v[at] = 0, 0
    q = torch.zeros(new, 2, dim, dtype=dtype)
    q[:, :, 0] = 8
    pages = np.arange(-(-n // 16))[None]
    plan = A.PagedPlan([new], [n], pages, n_pages=pages.size, page_size=16, q_heads=2, kv_heads=1,
                       head_dim=dim, units=1)
    out, lse = A.taps_attend(q.cuda(), paged(k, 16), paged(v, 16), plan, scale=0.125, lse=True)
    want, bound, w_lse, b_lse = R.attend(R.f64(q), R.f64(k), R.f64(v), n - new, 0, True, 0, 0.125,
                                         dtype)
    if dtype is F16:
        # that bound counts half a step of the smallest numbers, 2^-25, for every numerator, with
        # the largest at 1; at 2^10 they are 2^10 times as many steps, and all else stays
        seen = np.cumsum(np.abs(R.f64(v)), axis=0)[n - new:]   # by each token
        bound = bound - (1 + R.ROUND[F16]) * 2.0 ** -25 * (1 - 2.0 ** -10) * seen
        assert (bound > 0).all() and (bound < 0.05 * want).all()
    R.check(out, want, bound, "result")
    R.check(lse, w_lse, b_lse, "lse")


@pytest.mark.parametrize("new", [1, 40, 300])
def test_equal_weights_and_large_values(new):
    """Nothing overflows where all numerators are as large as any, nor where scores rise slowly."""
    n, dim = 3000, 128
    for rise in (0.0, 0.004, 0.03):   # of a score, from key to key
        k = torch.zeros(n, 1, dim, dtype=F16)
        k[:, 0, 0] = torch.arange(n) * rise
        v = torch.full((n, 1, dim), 60000.0, dtype=F16)
        q = torch.zeros(new, 1, dim, dtype=F16)
        q[:, 0, 0] = 8
        pages = np.arange(-(-n // 16))[None]
        plan = A.PagedPlan([new], [n], pages, n_pages=pages.size, page_size=16, q_heads=1,
                           kv_heads=1, head_dim=dim, units=1)
        out, lse = A.taps_attend(q.cuda(), paged(k, 16), paged(v, 16), plan, scale=0.125, lse=True)
        want, bound, w_lse, b_lse = R.attend(R.f64(q), R.f64(k), R.f64(v), n - new, 0, True, 0,
                                             0.125, F16)
        R.check(out, want, bound, f"rise {rise}")
        R.check(lse, w_lse, b_lse, f"lse, rise {rise}")


# ---------------------------------------------------------------------------
# gradients
# ---------------------------------------------------------------------------

def test_gradients_of_gradients_raise():
    """They are not computed; a penalty on a gradient must not lose its term silently."""
    g = gen_of(41)
    q = randn(g, 1, 5, 2, 64, dtype=F32).requires_grad_()
    w = randn(g, 64, dtype=F32).requires_grad_()
    table = A.rotation_table(5, 64)
    out, _ = A.norm_rotate(q, None, w, None, table)
    (first,) = torch.autograd.grad(out.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.square().sum().backward()
    out, _ = A.norm_rotate(q, None, w, None, table)
    (same,) = torch.autograd.grad(out.square().sum(), q)
    assert torch.equal(first, same) and not same.requires_grad


def test_the_backward_call_without_a_gradient_says_so():
    g = gen_of(43)
    args = [randn(g, 5, 2, 64) for _ in range(4)] + [randn(g, 64) for _ in range(2)]
    table = A.rotation_table(5, 64)
    want = A.taps_norm_rotate_backward(*args, table)
    assert not any(t.requires_grad for t in want)
    for which in range(6):
        mine = [x.clone() for x in args]
        mine[which].requires_grad_()
        for t, x in zip(A.taps_norm_rotate_backward(*mine, table), want):
            assert torch.equal(t, x)
            with pytest.raises(RuntimeError, match="taps_norm_rotate_backward has no gradient"):
                t.sum().backward()
        with torch.no_grad():
            assert not any(t.requires_grad for t in A.taps_norm_rotate_backward(*mine, table))
    dq, _, _, dkw = A.taps_norm_rotate_backward(args[0].requires_grad_(), None, args[2], None,
                                                args[4], None, table)
    assert dq.requires_grad and dkw is None


def test_calls_without_a_gradient_say_so():
    g = gen_of(42)
    q, k = (randn(g, 5, 2, 64) for _ in range(2))
    w = randn(g, 64)
    table = A.rotation_table(5, 64)
    cache = randn(g, 1, 2, 16, 64)
    plan = A.PagedPlan([5], [5], [[0]], n_pages=1, page_size=16, q_heads=2, kv_heads=2, head_dim=64)
    want = A.taps_norm_rotate(q, k, w, w, table)
    want_out, want_lse = A.taps_attend(q, cache, cache, plan, lse=True)
    assert not any(t.requires_grad for t in (*want, want_out, want_lse))
    for which in range(3):
        args = [q.clone(), k.clone(), w.clone()]
        args[which].requires_grad_()
        for t, x in zip(A.taps_norm_rotate(*args, w, table), want):
            assert torch.equal(t, x)
            with pytest.raises(RuntimeError, match="call norm_rotate"):
                t.sum().backward()
        with torch.no_grad():
            assert not any(t.requires_grad for t in A.taps_norm_rotate(*args, w, table))
    for which in range(3):
        args = [q.clone(), cache.clone(), cache.clone()]
        args[which].requires_grad_()
        out, lse = A.taps_attend(*args, plan, lse=True)
        assert torch.equal(out, want_out) and torch.equal(lse, want_lse)
        for t in (out, lse, A.taps_attend(*args, plan)):
            with pytest.raises(RuntimeError, match="taps_attend has no gradient"):
                t.sum().backward()
        mine = torch.empty_like(q)
        assert A.taps_attend(*args, plan, out=mine) is mine and not mine.requires_grad
        assert torch.equal(mine, want_out)


# ---------------------------------------------------------------------------
# infinite and NaN values that many rows see
# ---------------------------------------------------------------------------

def _values_case(new, n, heads, dim, page, dtype, options, seed=51):
    g = gen_of(seed)
    k, v = (torch.randn(n, heads, dim, generator=g).to(dtype) for _ in range(2))
    q = randn(g, new, 2 * heads, dim, dtype=dtype)
    pages = np.arange(-(-n // page))[None]
    plan = A.PagedPlan([new], [n], pages, n_pages=pages.size, page_size=page, q_heads=2 * heads,
                       kv_heads=heads, head_dim=dim, **options)
    return q, k, v, plan


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", [
    # new tokens, keys, heads, dim, page, options
    (4, 3001, 1, 128, 16, {}),                                  # narrow items, in pieces
    (7, 700, 2, 40, 16, {"window": 90}),
    (150, 150, 2, 64, 16, {}),
    (90, 333, 2, 96, 32, {"window": 70}),
    (200, 2000, 1, 128, 64, {"units": 4096}),                   # in pieces
    (300, 2700, 1, 128, 64, {"units": 1}),                      # 256 rows an item
    (300, 2900, 1, 80, 16, {"units": 1, "window": 1500}),
    (130, 400, 2, 64, 16, {"causal": False}),
    (60, 200, 2, 72, 16, {"kv_starts": [33]}),
])
@pytest.mark.parametrize("where", ["first", "everywhere", "a column"])
def test_infinite_values_that_many_rows_see(spec, dtype, where):
    new, n, heads, dim, page, options = spec
    say(f"[gpu] attend infinite values {spec} {dtype} {where}")
    q, k, v, plan = _values_case(*spec[:5], dtype, options)
    start = options.get("kv_starts", [0])[0]
    if where == "first":
        v[start, :, 3], v[start, :, dim - 1] = math.inf, math.nan
    elif where == "everywhere":
        at = torch.rand(v.shape, generator=gen_of(5)) < 3e-3
        v[at] = math.inf
        v[torch.rand(v.shape, generator=gen_of(6)) < 1e-3] = math.nan
    else:
        v[:, 0, 5] = -math.inf
    out, lse = A.taps_attend(q, paged(k, page), paged(v, page), plan, lse=True)
    with np.errstate(invalid="ignore"):
        want, bound, w_lse, b_lse = R.attend(
            R.f64(q), R.f64(k), R.f64(v), n - new, start, options.get("causal", True),
            options.get("window", 0), dim ** -0.5, dtype)
    got, odd = R.f64(out), ~np.isfinite(want)
    assert odd.any() or (where == "first" and "window" in options)   # there no row sees it
    assert np.array_equal(odd, ~np.isfinite(got)), "not the same outputs are finite"
    # an infinity whose weight is below the type's range may be NaN
    assert np.array_equal(got[odd & ~np.isnan(got)], want[odd & ~np.isnan(got)])
    assert np.isnan(got[np.isnan(want)]).all()
    R.check(np.where(odd, 0, got), np.where(odd, 0, want), np.where(odd, 0, bound), "finite")
    R.check(lse, w_lse, b_lse, "lse")


@pytest.mark.parametrize("new,n", [(2048, 2048), (512, 16384), (4, 16384)])
def test_infinite_values_cost_a_few_passes(new, n):
    """A value that has overflowed early in a document, and all of them: rows that are done again
    take the time of a few passes, not that of a key at a time (hundreds)."""
    q, k, v, plan = _values_case(new, n, 4, 128, 64, BF16, {})
    kc, vc = paged(k, 64), paged(v, 64)
    cases = [vc, vc.clone(), torch.full_like(vc, math.nan)]
    cases[1][0, :, 2, 7] = math.inf
    times = []
    for c in cases:
        A.taps_attend(q, kc, c, plan)
        best = math.inf
        for _ in range(3):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            A.taps_attend(q, kc, c, plan)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) * 1e3)
        times.append(best)
    say(f"[gpu] attend {new} over {n}: {times[0]:.0f} us, one infinite value {times[1]:.0f}, "
        f"all NaN {times[2]:.0f}")
    assert max(times[1:]) < 20 * times[0] + 100


@pytest.mark.parametrize("dim", [64, 128])
def test_a_few_tokens_take_a_tokens_time(dim):
    """Rows that pad a wavefront do not send it into the path that raises maxima, nor do tiles that
    all rows see: four tokens of one head over keys in one piece take what one takes."""
    n = 16384
    g = gen_of(61)
    k, v = (paged(torch.randn(n, 8, dim, generator=g).to(BF16), 64) for _ in range(2))
    pages = np.arange(n // 64)[None]
    plans = [A.PagedPlan([new], [n], pages, n_pages=pages.size, page_size=64, q_heads=8, kv_heads=8,
                         head_dim=dim, units=1) for new in (1, 4)]
    q = randn(g, 4, 8, dim)
    times = [math.inf, math.inf]
    for _ in range(10):
        for i, new in enumerate((1, 4)):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            for _ in range(5):
                A.taps_attend(q[:new], k, v, plans[i])
            b.record()
            b.synchronize()
            times[i] = min(times[i], a.elapsed_time(b) * 200)
    say(f"[gpu] attend 1 and 4 tokens over {n}, heads of {dim}: {times[0]:.1f} and {times[1]:.1f} us")
    assert times[1] < 1.2 * times[0]


# ---------------------------------------------------------------------------
# more workgroups than one dimension of a launch holds threads for
# ---------------------------------------------------------------------------

def test_norm_of_many_tokens():
    """2^24 workgroups of 256 threads: the same as in calls of fewer tokens."""
    tokens, heads, dim = (1 << 24) + 3, 4, 7
    gen = torch.Generator(device="cuda")
    gen.manual_seed(71)
    q = torch.randn(tokens, heads, dim, generator=gen, device="cuda", dtype=BF16)
    w = torch.randn(dim, generator=gen, device="cuda", dtype=BF16)
    say(f"[gpu] norm of {tokens} tokens")
    out, _ = A.taps_norm_rotate(q, None, w, None, None)
    for a in range(0, tokens, 5_000_000):
        part, _ = A.taps_norm_rotate(q[a:a + 5_000_000], None, w, None, None)
        assert torch.equal(out[a:a + 5_000_000], part)


def test_append_of_many_tokens():
    tokens, heads, dim, page = (1 << 24) + 3, 2, 7, 4096
    n_pages = -(-tokens // page)
    k, v = (torch.arange(tokens * heads * dim, device="cuda").remainder(m).view(tokens, heads, dim)
            .to(BF16) for m in (251, 241))
    caches = [torch.zeros(n_pages, page, heads, dim, dtype=BF16, device="cuda") for _ in range(2)]
    say(f"[gpu] append of {tokens} tokens")
    plan = A.PagedPlan([tokens], [tokens], np.arange(n_pages)[None], n_pages=n_pages, page_size=page,
                       q_heads=heads, kv_heads=heads, head_dim=dim)
    A.taps_cache_append(k, v, *(c.transpose(1, 2) for c in caches), plan)
    assert torch.equal(caches[0].flatten(0, 1)[:tokens], k)
    assert torch.equal(caches[1].flatten(0, 1)[:tokens], v)


def test_attention_of_many_items():
    """A token and 128 heads of each of 2^17 + 1 sequences, two of which have keys."""
    seqs, heads, dim = (1 << 17) + 1, 128, 8
    g = gen_of(73)
    k, v = (randn(g, 2, heads, 16, dim) for _ in range(2))
    kv = np.zeros(seqs, dtype=np.int32)
    kv[[5, seqs - 1]] = 9, 16
    pages = np.zeros((seqs, 1), dtype=np.int32)
    pages[5] = 1
    q = torch.zeros(seqs, heads, dim, dtype=BF16, device="cuda")
    q[[5, seqs - 1]] = randn(g, 2, heads, dim)
    say(f"[gpu] attend {seqs} sequences of {heads} heads")
    how = {"n_pages": 2, "page_size": 16, "q_heads": heads, "kv_heads": heads, "head_dim": dim}
    out = A.taps_attend(q, k, v, A.PagedPlan([1] * seqs, kv, pages, **how))
    want = A.taps_attend(q[[5, seqs - 1]], k, v, A.PagedPlan([1, 1], [9, 16], [[1], [0]], **how))
    assert torch.equal(out[[5, seqs - 1]], want) and want.isfinite().all()
    out[[5, seqs - 1]] = 0
    assert (out == 0).all()


# ---------------------------------------------------------------------------
# strides
# ---------------------------------------------------------------------------

def test_strides_of_axes_of_one_are_not_used():
    """One token, one head, one page: how far the next would be does not matter."""
    g = gen_of(81)

    def odd(t, axis):   # the same tensor with a stride of 8 n + 3 where its length is 1
        assert t.shape[axis] == 1
        strides = list(t.stride())
        strides[axis] = strides[axis] * 2 + 3
        return t.as_strided(t.shape, strides)
    q, one_head = randn(g, 1, 8, 64), randn(g, 5, 1, 64)
    cache, v = (randn(g, 3, 8, 16, 64) for _ in range(2))
    plan = A.PagedPlan([1], [40], [[2, 0, 1]], n_pages=3, page_size=16, q_heads=8, kv_heads=8,
                       head_dim=64)
    want = A.taps_attend(q, cache, v, plan)
    assert torch.equal(A.taps_attend(odd(q, 0), cache, v, plan), want)
    out = odd(torch.empty_like(q), 0)
    assert torch.equal(A.taps_attend(q, cache, v, plan, out=out), want)
    page, pv = (randn(g, 1, 1, 16, 64) for _ in range(2))
    plan = A.PagedPlan([5], [9], [[0]], n_pages=1, page_size=16, q_heads=1, kv_heads=1, head_dim=64)
    want = A.taps_attend(one_head, page, pv, plan)
    assert torch.equal(A.taps_attend(odd(one_head, 1), odd(page, 0), odd(odd(pv, 0), 1), plan), want)


def test_overlapping_tokens():
    """Queries that are a sliding window over one long row, by eight elements and by one."""
    g = gen_of(82)
    long, w, grad = randn(g, 1000), randn(g, 64), randn(g, 9, 4, 64)
    table = A.rotation_table(9, 64)
    cache, v = (randn(g, 1, 4, 16, 64) for _ in range(2))
    plan = A.PagedPlan([9], [9], [[0]], n_pages=1, page_size=16, q_heads=4, kv_heads=4, head_dim=64)
    for by in (8, 1):
        q = long.as_strided((9, 4, 64), (by, 72, 1))
        dense = q.contiguous()
        out, _ = A.taps_norm_rotate(q, None, w, None, table)
        assert torch.equal(out, A.taps_norm_rotate(dense, None, w, None, table)[0])
        got = A.taps_norm_rotate_backward(grad, None, q, None, w, None, table)
        want = A.taps_norm_rotate_backward(grad, None, dense, None, w, None, table)
        # not the same path: rows that start anywhere are read element by element
        b = 2 * R.ROUND[BF16] * want[0].abs().max() + 2e-5 * want[0].abs().max()
        assert (got[0] - want[0]).abs().max() <= b
        if by == 8:
            assert torch.equal(A.taps_attend(q, cache, v, plan),
                               A.taps_attend(dense, cache, v, plan))


# ---------------------------------------------------------------------------
# scores of minus infinity
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("spec", [
    # new tokens, keys, heads, dim, page, options
    (1, 4, 2, 64, 16, {}), (3, 6, 1, 128, 16, {}), (9, 9, 2, 96, 16, {}), (150, 150, 2, 64, 16, {}),
    (40, 4000, 1, 128, 64, {"units": 4096}),                    # in pieces
    (1, 9000, 1, 64, 64, {"units": 4096}),
    (2500, 2500, 1, 128, 64, {"units": 1}),                     # 256 rows an item
])
def test_scores_of_minus_infinity(spec, dtype):
    """Keys whose scores are all -inf weigh nothing beside others; a row that sees no others has
    no softmax and is NaN, unlike one that sees no key."""
    new, n, heads, dim, page, options = spec
    say(f"[gpu] attend scores of -inf {spec} {dtype}")
    q, k, v, plan = _values_case(new, n, heads, dim, page, dtype, options)
    q = q.abs()
    dead = {1: n, 3: 4, 40: 3000, 2500: 70}.get(new, 5)   # so many keys from the first on
    if n == 9000:
        dead = 8999
    k[:dead, :, 3] = -math.inf
    out, lse = A.taps_attend(q, paged(k, page), paged(v, page), plan, lse=True)
    gone = np.arange(n - new, n) < dead
    assert out[torch.from_numpy(gone).cuda()].isnan().all()
    assert lse[torch.from_numpy(gone).cuda()].isnan().all()
    if not gone.all():
        want, bound, w_lse, b_lse = R.attend(R.f64(q)[~gone], R.f64(k), R.f64(v),
                                             max(n - new, dead), dead, True, 0, dim ** -0.5, dtype)
        R.check(out[torch.from_numpy(~gone).cuda()], want, bound, "others")
        R.check(lse[torch.from_numpy(~gone).cuda()], w_lse, b_lse, "lse of others")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("new,n,heads,dim,options", [
    (20, 20, 40, 64, {}), (9, 200, 32, 128, {}), (3, 70, 64, 96, {"window": 9}),
    (40, 1500, 32, 128, {"units": 1}), (20, 3000, 40, 64, {"units": 4096}),
])
def test_infinite_values_and_many_heads(new, n, heads, dim, options, dtype):
    """A wavefront whose rows are all of one token, beside others of later tokens: what those see
    does not reach it."""
    say(f"[gpu] attend infinite values, {heads} heads {new} {n} {dim} {dtype}")
    g = gen_of(91)
    k, v = (torch.randn(n, 1, dim, generator=g).to(dtype) for _ in range(2))
    q = randn(g, new, heads, dim, dtype=dtype)
    pages = np.arange(-(-n // 16))[None]
    plan = A.PagedPlan([new], [n], pages, n_pages=pages.size, page_size=16, q_heads=heads,
                       kv_heads=1, head_dim=dim, **options)
    for j, value in ((1, math.inf), (new // 2, math.nan), (new - 2, -math.inf)):
        v[n - 1 - j, 0, (5 * j) % dim] = value
    out, lse = A.taps_attend(q, paged(k, 16), paged(v, 16), plan, lse=True)
    with np.errstate(invalid="ignore"):
        want, bound, w_lse, b_lse = R.attend(R.f64(q), R.f64(k), R.f64(v), n - new, 0, True,
                                             options.get("window", 0), dim ** -0.5, dtype)
    same_specials(out, want, np.nan_to_num(bound), "result")
    R.check(lse, w_lse, b_lse, "lse")
