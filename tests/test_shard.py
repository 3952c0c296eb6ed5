"""Shares of an attention block as strategies leave them, and one run on the GPU."""
import pytest

from paper_2301_04285_amd import shard, workloads as W


def test_share_of_a_strategy():
    op = W.attn_scores("scores", 8, 16, 1024, 64, 2)
    assert shard.share_of(op, (0, 0, 0, 0, 0)) == shard.Share(8, 16, 1024, 1024, 64)
    s = shard.share_of(op, (1, 2, 3, 0, 0))
    assert s == shard.Share(4, 4, 128, 1024, 64)
    # pairs of the last 128 of 1024 tokens, one by one
    assert s.flops == 4 * 64 * 4 * 4 * sum(range(1024 - 128 + 1, 1025))
    with pytest.raises(ValueError, match="not split"):
        shard.share_of(op, (0, 0, 0, 1, 0))
    with pytest.raises(ValueError, match="scores"):
        shard.share_of(W.softmax("softmax", 8, 16, 1024, 2), (0, 0, 0, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("share", [shard.Share(4, 4, 128, 1024, 64),   # a query chunk
                                   shard.Share(2, 2, 256, 256, 64),    # no split of the tokens
                                   shard.Share(3, 1, 1, 100, 128)])    # a single token
def test_share_runs(share):
    import torch
    seconds, difference = shard.run(share, torch.bfloat16, repeats=2)
    assert set(seconds) == {"norm_rotate", "gradients", "append", "attend"}
    # numerators and results rounded to 8 bits, each by up to 2^-8 of what they add up to, which
    # exceeds the largest result of a row by no more than a few times
    assert difference < 8 * 2.0 ** -8
