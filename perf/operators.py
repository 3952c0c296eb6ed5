"""The operators of one device's share of an attention block, sized for timing.

A strategy that splits the batch, head and query axes of a transformer's
attention leaves a device with some heads and a chunk of the tokens.  The
cases run what it does with them: norm and rotation of queries and keys
("norm_rotate", in training with its gradients), appending keys and values to
a paged cache ("append"), and attention of the new tokens over that cache
("attend").  With ``own`` the framework's kernels run, otherwise elementary
torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
BASE = 10000.0
MOST_FLOPS = 4 * 128 * 32 * 8 * (2048 * 2049 // 2)   # the listed prompts of eight sequences
MOST_BYTES = 540 * 10 ** 6


def listed():
    return [
        # eight sequences of the 4-layer GPT, one token each: all latency
        {"name": "norm_rotate gpt4 token", "op": "norm_rotate", "train": False, "dtype": "bf16",
         "batch": 8, "tokens": 1, "q_heads": 16, "k_heads": 16, "dim": 64, "rotary": 64,
         "interleaved": False, "packed": True},
        # a training step of the 24-layer GPT, batch 16 split over four devices
        {"name": "norm_rotate gpt24 train", "op": "norm_rotate", "train": True, "dtype": "bf16",
         "batch": 4, "tokens": 2048, "q_heads": 32, "k_heads": 32, "dim": 128, "rotary": 128,
         "interleaved": False, "packed": False},
        # documents packed end to end, grouped key heads, half of each head rotated, in pairs
        {"name": "norm_rotate packed train", "op": "norm_rotate", "train": True, "dtype": "fp16",
         "batch": 1, "tokens": 1531, "q_heads": 12, "k_heads": 4, "dim": 96, "rotary": 48,
         "interleaved": True, "packed": True},
        # one new token of each of 64 sequences
        {"name": "append 64 tokens", "op": "append", "dtype": "fp16", "seqs": 64, "new": 1,
         "old": 120, "spread": True, "kv_heads": 32, "dim": 128, "rotary": 128,
         "interleaved": False, "norm": False, "page": 16},
        # the prompts of eight sequences of the 24-layer GPT, keys normed on the way
        {"name": "append gpt24 prompts", "op": "append", "dtype": "bf16", "seqs": 8, "new": 2048,
         "old": 0, "spread": False, "kv_heads": 32, "dim": 128, "rotary": 128,
         "interleaved": False, "norm": True, "page": 64},
        # one token of one sequence of the 4-layer GPT: latency
        {"name": "attend gpt4 token", "op": "attend", "dtype": "bf16", "seqs": 1, "chunks": 0,
         "new": 1, "kv": 1024, "spread": False, "q_heads": 16, "kv_heads": 16, "dim": 64,
         "window": 0, "page": 16},
        # a serving batch: 64 sequences of different lengths, four query heads to a key head
        {"name": "attend 64 tokens", "op": "attend", "dtype": "bf16", "seqs": 64, "chunks": 0,
         "new": 1, "kv": 4000, "spread": True, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "window": 0, "page": 64},
        # two long documents, one token each: the cache is what there is to read
        {"name": "attend long tokens", "op": "attend", "dtype": "bf16", "seqs": 2, "chunks": 0,
         "new": 1, "kv": 131001, "spread": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "window": 0, "page": 64},
        # the prompts of eight sequences of the 24-layer GPT: the most products
        {"name": "attend gpt24 prompts", "op": "attend", "dtype": "bf16", "seqs": 8, "chunks": 8,
         "new": 2048, "kv": 2048, "spread": False, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "window": 0, "page": 64},
        # the query chunk that a split of the sequence axis leaves, late in a long document
        {"name": "attend chunk of 512", "op": "attend", "dtype": "bf16", "seqs": 1, "chunks": 1,
         "new": 512, "kv": 32768, "spread": False, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "window": 0, "page": 64},
        # prompts and single tokens in one call, a sliding window, odd lengths
        {"name": "attend mixed window", "op": "attend", "dtype": "fp16", "seqs": 21, "chunks": 2,
         "new": 701, "kv": 3001, "spread": True, "q_heads": 12, "kv_heads": 4, "dim": 96,
         "window": 1000, "page": 16},
        # the 4-layer GPT's prompts, small heads
        {"name": "attend gpt4 prompts", "op": "attend", "dtype": "fp16", "seqs": 8, "chunks": 8,
         "new": 1024, "kv": 1024, "spread": False, "q_heads": 16, "kv_heads": 16, "dim": 64,
         "window": 0, "page": 16},
    ]


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return case


def _draw(rng):
    def log_int(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    op = rng.choice(("norm_rotate", "append", "attend", "attend"))
    kv_heads = rng.choice((1, 2, 4, 8, 12, 16, 32))
    q_heads = kv_heads * rng.choice((1, 1, 2, 4, 8))
    dim = rng.choice((64, 64, 80, 96, 128, 128, 128))
    if op == "norm_rotate":
        return {"op": op, "train": rng.random() < 0.6, "dtype": rng.choice(("bf16", "fp16", "fp32")),
                "batch": log_int(1, 16), "tokens": log_int(1, 4096), "q_heads": q_heads,
                "k_heads": kv_heads, "dim": dim, "rotary": rng.choice((dim, dim, dim // 2)),
                "interleaved": rng.random() < 0.3, "packed": rng.random() < 0.5}
    page = rng.choice((16, 32, 64, 128))
    dtype = rng.choice(("bf16", "fp16"))
    if op == "append":
        return {"op": op, "dtype": dtype, "seqs": log_int(1, 128), "new": log_int(1, 4096),
                "old": rng.choice((0, log_int(1, 500))), "spread": rng.random() < 0.5,
                "kv_heads": kv_heads, "dim": dim, "rotary": rng.choice((dim, dim, dim // 2)),
                "interleaved": rng.random() < 0.3, "norm": rng.random() < 0.5, "page": page}
    seqs = log_int(1, 128)
    chunks = rng.choice((0, seqs, max(1, seqs // 8)))
    new = log_int(2, 2048) if chunks else rng.choice((1, 1, 1, 2, 4))
    return {"op": op, "dtype": dtype, "seqs": seqs, "chunks": chunks, "new": new,
            "kv": new + (rng.choice((0, log_int(1, 131072))) if chunks else log_int(1, 131072)),
            "spread": rng.random() < 0.6,
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "window": rng.choice((0, 0, 0, log_int(64, 4096))), "page": page}


# ---------------------------------------------------------------------------
# lengths and inputs
# ---------------------------------------------------------------------------

def _key(case):
    return str(sorted((k, v) for k, v in case.items() if k != "name"))


def _lengths(case):
    """(new tokens, keys after them) per sequence; "spread": from an eighth of the case's length
    up to it."""
    r = random.Random(_key(case))
    q_lens, kv_lens = [], []
    for s in range(case["seqs"]):
        if case["op"] == "append":
            old = r.randint(case["old"] // 8, case["old"]) if case["spread"] else case["old"]
            new = max(1, r.randint(case["new"] // 8, case["new"])) if case["spread"] else case["new"]
            q_lens.append(new)
            kv_lens.append(old + new)
        else:
            new = case["new"] if s < case["chunks"] or not case["chunks"] else 1
            kv = max(1, r.randint(case["kv"] // 8, case["kv"])) if case["spread"] else case["kv"]
            new = min(new, kv)
            q_lens.append(new)
            kv_lens.append(kv)
    return q_lens, kv_lens


def _pages(case, kv_lens, seed):
    """A page table [sequences, most pages] (-1: none) over the pages in a random order, and their
    number: one more than the sequences need."""
    counts = [-(-n // case["page"]) for n in kv_lens]
    order = list(range(sum(counts) + 1))
    random.Random("%d %s" % (seed, _key(case))).shuffle(order)
    table = np.full((len(counts), max(counts)), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    return table, len(order)


def _randn(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _weight(gen, dim, dtype):
    return (1 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(dtype)


def _table(n_positions, rotary):
    """cos and sin of position x base^(-2 i / rotary), [positions, 2, rotary / 2]."""
    inv = BASE ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    angle = torch.arange(n_positions, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.stack((angle.cos(), angle.sin()), dim=1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(random.Random("%d %s" % (seed, _key(case))).getrandbits(48))
    dtype = DTYPES[case["dtype"]]
    state = {"case": case}
    if case["op"] == "norm_rotate":
        shape = (case["batch"], case["tokens"])
        # as one projection leaves them side by side
        both = _randn(gen, (*shape, case["q_heads"] + case["k_heads"], case["dim"]), dtype, 2.0)
        state["q"], state["k"] = both.split((case["q_heads"], case["k_heads"]), dim=2)
        state["q_weight"] = _weight(gen, case["dim"], dtype)
        state["k_weight"] = _weight(gen, case["dim"], dtype)
        n_positions = 4096
        state["table"] = _table(n_positions, case["rotary"])
        state["first"] = random.Random(seed).randrange(n_positions - case["tokens"] + 1)
        state["positions"] = None
        if case["packed"]:   # every token its own position
            state["positions"] = torch.randint(n_positions, shape, generator=gen, device="cuda",
                                               dtype=torch.int32)
        if case["train"]:
            state["dq"] = _randn(gen, state["q"].shape, dtype)
            state["dk"] = _randn(gen, state["k"].shape, dtype)
        return state
    q_lens, kv_lens = _lengths(case)
    pages, n_pages = _pages(case, kv_lens, seed)
    tokens, shape = sum(q_lens), (n_pages, case["kv_heads"], case["page"], case["dim"])
    state.update(q_lens=q_lens, kv_lens=kv_lens, pages=pages)
    if case["op"] == "append":
        state["k"] = _randn(gen, (tokens, case["kv_heads"], case["dim"]), dtype, 2.0)
        state["v"] = _randn(gen, (tokens, case["kv_heads"], case["dim"]), dtype)
        state["k_weight"] = _weight(gen, case["dim"], dtype) if case["norm"] else None
        state["table"] = _table(max(kv_lens), case["rotary"])
        state["k_cache"], state["v_cache"] = (_randn(gen, shape, dtype) for _ in range(2))
    else:
        state["q"] = _randn(gen, (tokens, case["q_heads"], case["dim"]), dtype)
        state["k_cache"], state["v_cache"] = (_randn(gen, shape, dtype) for _ in range(2))
        _spoil(case, state, pages, kv_lens)
    if own:
        from paper_2301_04285_amd import attention
        state["plan"] = attention.PagedPlan(
            q_lens, kv_lens, pages, n_pages=n_pages, page_size=case["page"],
            q_heads=case.get("q_heads", case["kv_heads"]), kv_heads=case["kv_heads"],
            head_dim=case["dim"], window=case.get("window", 0))
    else:
        state["slots"] = [_slots(case, pages[s], n) for s, n in enumerate(kv_lens)]
    return state


def _slots(case, row, n):
    """(page, slot) of keys 0 .. n - 1 of a sequence, on the GPU."""
    at = torch.arange(n, device="cuda")
    return torch.from_numpy(row).cuda().long()[at // case["page"]], at % case["page"]


def _spoil(case, state, pages, kv_lens):
    """Slots that no key has been written to hold what memory held before: NaN here."""
    free = torch.ones(state["k_cache"].shape[0], case["page"], dtype=torch.bool, device="cuda")
    for s, n in enumerate(kv_lens):
        free[_slots(case, pages[s], n)] = False
    for c in ("k_cache", "v_cache"):
        state[c].masked_fill_(free[:, None, :, None], float("nan"))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)[case["op"]](state, case)


def _own_norm_rotate(state, case):
    from paper_2301_04285_amd import attention
    args = (state["q"], state["k"], state["q_weight"], state["k_weight"], state["table"])
    how = {"positions": state["positions"], "first": state["first"], "eps": EPS,
           "interleaved": case["interleaved"]}
    q_out, k_out = attention.taps_norm_rotate(*args, **how)
    if not case["train"]:
        return {"q": q_out, "k": k_out}
    grads = attention.taps_norm_rotate_backward(state["dq"], state["dk"], *args, **how)
    return {"q": q_out, "k": k_out, "grads": list(grads)}


def _own_append(state, case):
    from paper_2301_04285_amd import attention
    attention.taps_cache_append(state["k"], state["v"], state["k_cache"], state["v_cache"],
                                state["plan"], table=state["table"], k_weight=state["k_weight"],
                                eps=EPS, interleaved=case["interleaved"])
    return {"k": state["k_cache"], "v": state["v_cache"]}


def _own_attend(state, case):
    from paper_2301_04285_amd import attention
    return attention.taps_attend(state["q"], state["k_cache"], state["v_cache"], state["plan"])


_run_own = {"norm_rotate": _own_norm_rotate, "append": _own_append, "attend": _own_attend}


def _pair(x, rotary, interleaved):
    """The two members of every rotated pair, and what is not rotated."""
    if interleaved:
        return x[..., 0:rotary:2], x[..., 1:rotary:2], x[..., rotary:]
    return x[..., :rotary // 2], x[..., rotary // 2:rotary], x[..., rotary:]


def _unpair(a, b, rest, interleaved):
    if interleaved:
        return torch.cat((torch.stack((a, b), dim=-1).flatten(-2), rest), dim=-1)
    return torch.cat((a, b, rest), dim=-1)


def _rows(state, case):
    """cos and sin of every token, to broadcast over its heads."""
    if state["positions"] is not None:
        rows = state["table"][state["positions"].long()]
    else:
        rows = state["table"][state["first"]:state["first"] + case["tokens"]][None]
    return rows[:, :, None, 0], rows[:, :, None, 1]


def _rstd(x):
    return torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)


def _norm_rotate(x, w, c, s, case):
    n = x if w is None else x * _rstd(x) * w
    a, b, rest = _pair(n, case["rotary"], case["interleaved"])
    return _unpair(a * c - b * s, b * c + a * s, rest, case["interleaved"])


def _norm_rotate_gradients(g, x, w, c, s, case):
    a, b, rest = _pair(g, case["rotary"], case["interleaved"])
    h = _unpair(a * c + b * s, b * c - a * s, rest, case["interleaved"])
    rstd = _rstd(x)
    xh = x * rstd
    dw = (h * xh).flatten(0, -2).sum(dim=0)
    h = h * w
    return rstd * (h - xh * (h * xh).mean(dim=-1, keepdim=True)), dw


def _plain_norm_rotate(state, case):
    c, s = _rows(state, case)
    dtype, out, grads = state["q"].dtype, {}, {}
    for side in "qk":
        x, w = state[side].float(), state[side + "_weight"].float()
        out[side] = _norm_rotate(x, w, c, s, case).to(dtype)
        if case["train"]:
            grads[side] = _norm_rotate_gradients(state["d" + side].float(), x, w, c, s, case)
    if case["train"]:
        out["grads"] = [grads[side][n].to(dtype) for n in range(2) for side in "qk"]
    return out


def _plain_append(state, case):
    dtype, at = state["k"].dtype, 0
    w = None if state["k_weight"] is None else state["k_weight"].float()
    for new, kv, (page, slot) in zip(state["q_lens"], state["kv_lens"], state["slots"]):
        rows = state["table"][kv - new:kv]
        k = _norm_rotate(state["k"][at:at + new].float(), w, rows[:, None, 0], rows[:, None, 1],
                         case)
        state["k_cache"][page[kv - new:], :, slot[kv - new:]] = k.to(dtype)
        state["v_cache"][page[kv - new:], :, slot[kv - new:]] = state["v"][at:at + new]
        at += new
    return {"k": state["k_cache"], "v": state["v_cache"]}


def _plain_attend(state, case):
    q_all, at = state["q"], 0
    group = case["q_heads"] // case["kv_heads"]
    out = torch.empty_like(q_all)
    for new, kv, (page, slot) in zip(state["q_lens"], state["kv_lens"], state["slots"]):
        first = max(0, kv - new + 1 - case["window"]) if case["window"] else 0
        page, slot = page[first:], slot[first:]
        keys = state["k_cache"][page, :, slot].float().permute(1, 2, 0).contiguous()
        values = state["v_cache"][page, :, slot].float().transpose(0, 1).contiguous()
        q = q_all[at:at + new].float().view(new, case["kv_heads"], group, case["dim"])
        q = q.permute(1, 2, 0, 3).reshape(case["kv_heads"], group * new, case["dim"])
        p = torch.arange(kv - new, kv, device="cuda")[:, None]
        j = torch.arange(first, kv, device="cuda")[None]
        hidden = j > p
        if case["window"]:
            hidden = hidden | (j <= p - case["window"])
        hidden = hidden.repeat(group, 1)
        most = max(1, (1 << 29) // (group * new * (kv - first)))   # heads at a time: 2 GiB of scores
        for h in range(0, case["kv_heads"], most):
            s = torch.matmul(q[h:h + most] * case["dim"] ** -0.5, keys[h:h + most])
            s = s.masked_fill_(hidden, float("-inf"))
            s = torch.exp(s - s.amax(dim=-1, keepdim=True))
            o = torch.matmul(s, values[h:h + most]) / s.sum(dim=-1, keepdim=True)
            o = o.view(-1, group, new, case["dim"]).permute(2, 0, 1, 3).flatten(1, 2)
            out[at:at + new, h * group:h * group + o.shape[1]] = o.to(out.dtype)
        at += new
    return out


_run_plain = {"norm_rotate": _plain_norm_rotate, "append": _plain_append, "attend": _plain_attend}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _visible(case, new, kv):
    """Pairs of a query and a key it sees, and the keys that any query sees."""
    w = case["window"] or kv
    first = kv - new   # the first query's position: it sees min(w, first + 1) keys
    short = max(0, min(new, w - first - 1))   # queries that see fewer than w
    pairs = short * (first + 1) + short * (short - 1) // 2 + (new - short) * w
    return pairs, kv - max(0, first + 1 - w)


def work(case):
    """Inputs read once, outputs written once.  Norm and rotation are some ten operations an
    element, as many again for the gradients; attention two products a visible pair."""
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "norm_rotate":
        tokens = case["batch"] * case["tokens"]
        n = tokens * (case["q_heads"] + case["k_heads"]) * case["dim"]
        rows = (tokens if case["packed"] else case["tokens"]) * 4 * case["rotary"]
        if case["train"]:
            return {"bytes": 4 * n * size + rows + 8 * case["dim"] * size, "flops": 24 * n}
        return {"bytes": 2 * n * size + rows + 2 * case["dim"] * size, "flops": 8 * n}
    q_lens, kv_lens = _lengths(case)
    if case["op"] == "append":
        n = sum(q_lens) * case["kv_heads"] * case["dim"]
        return {"bytes": 4 * n * size + sum(q_lens) * 4 * case["rotary"],
                "flops": (8 if case["norm"] else 4) * n}
    pairs, keys = (sum(x) for x in zip(*(_visible(case, *s) for s in zip(q_lens, kv_lens))))
    return {"bytes": 2 * size * case["dim"] * (sum(q_lens) * case["q_heads"]
                                               + keys * case["kv_heads"]),
            "flops": 4 * case["dim"] * case["q_heads"] * pairs}


# ---------------------------------------------------------------------------
# in 64 bits from the definitions
# ---------------------------------------------------------------------------

def _rotation(cos, sin, case):
    """The rotation of a head as matrices [..., dim, dim]: y = R n."""
    dim, half = case["dim"], case["rotary"] // 2
    r = torch.zeros((*cos.shape[:-1], dim, dim), dtype=torch.float64, device="cuda")
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        r[..., a, a] = r[..., b, b] = cos[..., i]
        r[..., a, b] = -sin[..., i]
        r[..., b, a] = sin[..., i]
    for i in range(2 * half, dim):
        r[..., i, i] = 1
    return r


def _exact_rows(x, w, cos, sin, case, g=None):
    """x, g [rows, heads, dim]; cos, sin [rows, ...]: y, and with g the gradients from the
    Jacobian of the norm."""
    r = _rotation(cos.double(), sin.double(), case)
    x = x.double()
    if w is None:
        return (r @ x.transpose(1, 2)).transpose(1, 2)
    w = w.double()
    length = (x.square().sum(dim=-1, keepdim=True) / case["dim"] + EPS).sqrt()
    y = ((r * w) @ (x / length).transpose(1, 2)).transpose(1, 2)
    if g is None:
        return y
    h = g.double() @ r               # rows of R^T g
    dw = (h * x / length).sum(dim=(0, 1))
    hw = h * w
    dx = hw / length - x * (hw * x).sum(dim=-1, keepdim=True) / (case["dim"] * length ** 3)
    return y, dx, dw


def _exact_norm_rotate(state, case):
    tokens = case["batch"] * case["tokens"]
    if state["positions"] is not None:
        rows = state["table"][state["positions"].long().view(-1)]
    else:
        rows = state["table"][state["first"]:state["first"] + case["tokens"]]
        rows = rows.repeat(case["batch"], 1, 1)
    out, grads = {}, {}
    for side in "qk":
        x, w = state[side].flatten(0, 1), state[side + "_weight"]
        g = state["d" + side].flatten(0, 1) if case["train"] else None
        parts, dw = [], 0
        for a in range(0, tokens, 512):
            b = min(tokens, a + 512)
            part = _exact_rows(x[a:b], w, rows[a:b, 0], rows[a:b, 1], case,
                               None if g is None else g[a:b])
            if case["train"]:
                dw = dw + part[2]
                parts.append(part[:2])
            else:
                parts.append((part,))
        out[side] = torch.cat([p[0] for p in parts]).view(state[side].shape)
        if case["train"]:
            grads[side] = torch.cat([p[1] for p in parts]).view(state[side].shape), dw
    if case["train"]:
        out["grads"] = [grads[side][n] for n in range(2) for side in "qk"]
    return out


def _exact_append(state, case):
    k_cache, v_cache = state["k_cache"].double(), state["v_cache"].double()
    at = 0
    for s, (new, kv) in enumerate(zip(state["q_lens"], state["kv_lens"])):
        for a in range(kv - new, kv, 512):
            p = torch.arange(a, min(kv, a + 512), device="cuda")
            i = at + p - (kv - new)
            page = torch.as_tensor(state["pages"][s], device="cuda").long()[p // case["page"]]
            rows = state["table"][p]
            k_cache[page, :, p % case["page"]] = _exact_rows(
                state["k"][i], state["k_weight"], rows[:, 0], rows[:, 1], case)
            v_cache[page, :, p % case["page"]] = state["v"][i].double()
        at += new
    return {"k": k_cache, "v": v_cache}


def _exact_attend(state, case):
    """Block by block over the keys, with the largest score of every row known beforehand."""
    q = state["q"].double() / math.sqrt(case["dim"])
    out, at = torch.zeros_like(q), 0
    for s, (new, kv) in enumerate(zip(state["q_lens"], state["kv_lens"])):
        row = torch.as_tensor(state["pages"][s], device="cuda").long()
        for h in range(case["q_heads"]):
            head = h // (case["q_heads"] // case["kv_heads"])
            mine = q[at:at + new, h]
            blocks = []
            for a in range(0, kv, 8192):
                j = torch.arange(a, min(kv, a + 8192), device="cuda")
                i = torch.arange(new, device="cuda")[:, None] + (kv - new)
                seen = (j <= i) if not case["window"] else (j <= i) & (i - j < case["window"])
                if not bool(seen.any()):
                    continue
                page, slot = row[j // case["page"]], j % case["page"]
                score = mine @ state["k_cache"][page, head, slot].double().T
                blocks.append((torch.where(seen, score, -math.inf),
                               state["v_cache"][page, head, slot].double()))
            top = torch.stack([b.max(dim=1).values for b, _ in blocks]).max(dim=0).values
            weights = [(b - top[:, None]).exp() for b, _ in blocks]
            total = sum(w.sum(dim=1) for w in weights)
            out[at:at + new, h] = sum(w @ v for w, (_, v) in zip(weights, blocks)) / total[:, None]
        at += new
    return out


def exact(case, seed):
    if case["op"] == "attend" and (case["seqs"] * case["q_heads"] > 2048
                                   or case["seqs"] * case["q_heads"] * case["kv"] > 1 << 25):
        return None   # thousands of products and more
    state = prepare(case, seed)
    return {"norm_rotate": _exact_norm_rotate, "append": _exact_append,
            "attend": _exact_attend}[case["op"]](state, case)
