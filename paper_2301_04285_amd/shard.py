"""One device's share of an attention block, as a plan splits it, run and timed.

``python -m paper_2301_04285_amd.shard`` searches a transformer layer's plan over the cost
tables (``search.solve`` on t), reads from it how the attention scores are split -- a
strategy may cut the batch, the heads and the query tokens, never the keys -- and
runs the share of the device that holds the last tokens, whose queries see the
most keys: the earlier tokens' keys are in a paged cache; the chunk's queries are
normed and rotated, its keys and values appended on the way, and attended.  The
printed times stand beside the communication seconds that the plan was chosen by.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

__all__ = ["Share", "share_of", "run"]

PAGE = 64


@dataclass(frozen=True)
class Share:
    """Sequences, heads and tokens of one device, and the sequence's keys."""
    batch: int
    heads: int
    tokens: int
    keys: int
    dim: int

    @property
    def flops(self) -> int:
        """Two products per query head and visible pair, for the last tokens."""
        first = self.keys - self.tokens + 1
        pairs = self.tokens * (first + self.keys) // 2
        return 4 * self.dim * self.batch * self.heads * pairs


def share_of(op, log2_degrees) -> Share:
    """What a strategy of a ``scores`` operator (workloads.attn_scores: axes b, n, s, t, d)
    leaves to one device; log2_degrees: the strategy's, per axis."""
    if op.kind != "scores" or op.axis_names != ("b", "n", "s", "t", "d"):
        raise ValueError(f"{op.name} does not compute attention scores")
    length = [n >> int(d) for n, d in zip(op.axis_len, log2_degrees)]
    b, n, s, t, d = length
    if t != op.axis_len[3] or d != op.axis_len[4]:
        raise ValueError("keys and head dimension are not split")
    return Share(b, n, s, t, d)


def _slots(share: Share):
    """A page table for the share's sequences, one after the other, and its pages."""
    per_seq = -(-share.keys // PAGE)
    return np.arange(share.batch * per_seq, dtype=np.int32).reshape(share.batch, per_seq), \
        share.batch * per_seq


def run(share: Share, dtype, repeats: int = 10, seed: int = 0):
    """Runs the share on random projections; {step: seconds} and the largest difference
    of a few rows from 64-bit attention over the same cache, relative to it."""
    import torch

    from . import attention
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)
    b, n, new, keys, dim = share.batch, share.heads, share.tokens, share.keys, share.dim
    old = keys - new
    pages, n_pages = _slots(share)
    shape = {"n_pages": n_pages, "page_size": PAGE, "q_heads": n, "kv_heads": n, "head_dim": dim}
    table = attention.rotation_table(keys, dim)
    q_weight, k_weight = (1 + 0.1 * randn(dim) for _ in range(2))
    q, k, v = randn(b * new, 3 * n, dim).split(n, dim=1)   # as one projection leaves them
    caches = [torch.zeros((n_pages, n, PAGE, dim), dtype=dtype, device="cuda") for _ in range(2)]
    if old:   # the earlier chunks' keys, which other devices projected
        before = attention.PagedPlan([old] * b, [old] * b, pages, **shape)
        attention.taps_cache_append(randn(b * old, n, dim), randn(b * old, n, dim), *caches, before,
                                    table=table, k_weight=k_weight)
    plan = attention.PagedPlan([new] * b, [keys] * b, pages, **shape)
    chunk = q.unflatten(0, (b, new))
    state = {}

    def norm_rotate():
        state["q"], _ = attention.taps_norm_rotate(chunk, None, q_weight, None, table, first=old)

    def gradients():
        attention.taps_norm_rotate_backward(state["q"], None, chunk, None, q_weight, None, table,
                                            first=old)

    def append():
        attention.taps_cache_append(k, v, *caches, plan, table=table, k_weight=k_weight)

    def attend():
        state["out"] = attention.taps_attend(state["q"].flatten(0, 1), *caches, plan)
    seconds = {}
    for step in (norm_rotate, gradients, append, attend):
        step()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(repeats):
            step()
        end.record()
        end.synchronize()
        seconds[step.__name__] = start.elapsed_time(end) * 1e-3 / repeats
    return seconds, _difference(share, state, caches, pages)


def _difference(share: Share, state, caches, pages) -> float:
    worst = 0.0
    rng = np.random.default_rng(1)
    for _ in range(4):
        s, t, h = (int(rng.integers(x)) for x in (share.batch, share.tokens, share.heads))
        seen = share.keys - share.tokens + t + 1
        k, v = (c[pages[s], h].flatten(0, 1)[:seen].double().cpu().numpy() for c in caches)
        q = state["q"][s, t, h].double().cpu().numpy()
        p = k @ q * share.dim ** -0.5
        p = np.exp(p - p.max())
        want = p @ v / p.sum()
        got = state["out"].unflatten(0, (share.batch, share.tokens))[s, t, h].double().cpu().numpy()
        worst = max(worst, float(np.abs(got - want).max() / np.abs(want).max()))
    return worst


def main() -> int:
    import argparse
    import json
    import sys

    ap = argparse.ArgumentParser(description="one device's share of a transformer layer's "
                                             "attention, as the cheapest plan splits it")
    ap.add_argument("--config", type=int, default=3, choices=(2, 3, 5),
                    help="workloads.config of the transformer (one layer is planned)")
    ap.add_argument("--repeats", type=int, default=10)
    ap.add_argument("--time-limit", type=float, default=300.0, help="seconds for the ILP")
    args = ap.parse_args()

    import torch

    from . import search, taps, workloads as W

    if not torch.cuda.is_available():
        print("the tables are built and the share is run on a GPU", file=sys.stderr)
        return 1
    w = W.config(args.config)
    name, cluster = w.clusters[0]
    graph = W.leading_ops(w.graph, 14)
    tables = taps.build_tables(graph, cluster)
    torch.cuda.synchronize()
    node, edge = search.host_tables(graph, tables, "t")
    plan = search.solve(graph, node, edge, args.time_limit)
    scores = next(k for k, op in enumerate(graph.ops) if op.kind == "scores")
    log2_degrees, _ = taps.strategies_to_numpy(tables.strategies)
    op = graph.ops[scores]
    share = share_of(op, log2_degrees[int(tables.op_offsets[scores]) + plan.choice[scores]]
                     [:op.n_axes])
    dtype = torch.float16 if "fp16" in w.name else torch.bfloat16
    seconds, difference = run(share, dtype, args.repeats)
    print(json.dumps({
        "workload": f"{w.name} / {name}", "plan_communication_s": plan.objective,
        "share": {"sequences": share.batch, "heads": share.heads, "query_tokens": share.tokens,
                  "keys": share.keys, "head_dim": share.dim},
        "seconds": seconds, "attend_tflops": share.flops / seconds["attend"] * 1e-12,
        "difference": difference}), flush=True)
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
