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


def test_pieces(monkeypatch):
    """Together they are all positions, each no larger than it may be but for a single one."""
    for n_keys, most, steps in ((1000, 1 << 28, 1), (1000, 2 * 3 * 64 * 100, 10),
                                (1001, 2 * 3 * 64 * 100, 11), (7, 1, 7), (0, 100, 0)):
        monkeypatch.setattr(shard, "PIECE", most)
        pieces = shard._pieces(shard.Share(2, 3, 1, n_keys, 64), n_keys)
        assert len(pieces) == steps
        assert [j for first, end in pieces for j in range(first, end)] == list(range(n_keys))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 8, 16])
def test_share_needs_its_cache_and_little_more(bits, monkeypatch):
    """No step holds all keys and values beside the cache, neither in 32 bits nor in 16."""
    import torch
    share, piece = shard.Share(2, 8, 1, 32768, 128), 1 << 22
    monkeypatch.setattr(shard, "PIECE", piece)
    elements = share.batch * share.heads * share.keys * share.dim
    held = 2 * elements * (2 if bits == 16 else bits / 8 + 1 / 32)
    table = share.keys * share.dim * 4
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    _, difference = shard.run(share, torch.bfloat16, repeats=1, cache_bits=bits)
    # of a piece: keys in 16 bits, values in 32 and in 16; as much again for page tables, slots
    # and the allocator's roundings
    assert torch.cuda.max_memory_allocated() - before < held + table + 16 * piece
    assert difference < 8 * 2.0 ** -8
