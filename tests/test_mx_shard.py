"""One device's share of attention over a cache in a microscaling format."""
import pytest

from paper_2301_04285_amd import shard


def test_cache_bits_refusals():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="cache of 5 bits"):
        shard.run(shard.Share(1, 1, 1, 1, 64), torch.bfloat16, cache_bits=5)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("share", [shard.Share(4, 4, 128, 1024, 64),   # a query chunk
                                   shard.Share(2, 2, 256, 256, 64),    # no split of the tokens
                                   shard.Share(3, 1, 1, 100, 128)])    # a single token
def test_share_runs(share, bits):
    import torch
    seconds, difference = shard.run(share, torch.bfloat16, repeats=2, cache_bits=bits)
    assert set(seconds) == {"norm_rotate", "gradients", "append", "attend", "read"}
    # numerators and results rounded to 8 bits, each by up to 2^-8 of what they add up to, which
    # exceeds the largest result of a row by no more than a few times
    assert difference < 8 * 2.0 ** -8
