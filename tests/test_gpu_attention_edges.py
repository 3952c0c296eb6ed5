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
