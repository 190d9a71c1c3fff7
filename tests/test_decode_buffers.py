"""The buffers that PagedDecode keeps, on the CPU: their sizes are host code."""
import os
import shutil

import pytest


@pytest.fixture(scope="module")
def ssd():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2606_20543_gb300 import build
    build.build()
    import paper_2606_20543_gb300 as m
    m.load()
    return m


@pytest.fixture(autouse=True)
def sharing(ssd):
    yield
    ssd.load().ssd_set_cache_sharing(0)


def make(groups, max_shared, B=4, max_blocks=200):
    """A decoder without the tensors that only a GPU fills."""
    from paper_2606_20543_gb300.decode import PagedDecode
    dec = PagedDecode.__new__(PagedDecode)
    dec.__dict__.update(B=B, Hq=8, Hkv=2, d=128, block=16, max_blocks=max_blocks, device="cpu", groups=groups,
                        max_shared=max_shared, _ws={}, _outgrown=[])
    return dec


def test_the_workspace_follows_the_switch_whoever_sets_it(ssd):
    so, dec = ssd.load(), make(2, 90)
    need = lambda: so.ssd_cache_attention_shared_workspace(4, 2, 8, 2, 128, 1, 3200, 1440)  # noqa: E731
    assert ssd.ssd_get_cache_sharing() == 0
    sizes = []
    for how in (2, 1, 0, 1):
        assert so.ssd_set_cache_sharing(how) == 0  # (as a caller of the C library does)
        assert ssd.ssd_get_cache_sharing() == how
        ws, n = dec._workspace(1)
        assert n >= need() and n == ws.numel()
        sizes.append(need())
    assert sizes[1] > sizes[0]


def state(dec, num_blocks):
    """The tensors that share() and release() work on, of a pool that nothing holds."""
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    dec.__dict__.update(num_blocks=num_blocks, block_table=i32(dec.B, dec.max_blocks).fill_(-1),
                        cache_len=i32(dec.B), held=i32(dec.B), status=i32(1),
                        ring=torch.arange(num_blocks + 1, dtype=torch.int32),
                        head=torch.zeros(1, dtype=torch.int64), tail=torch.full((1,), num_blocks), _groups={},
                        _base=i32(dec.B), _open=i32(dec.B).fill_(1))
    return dec


def cached(dec, b, tokens):
    """Sequence b caches `tokens` tokens in the pool's next blocks."""
    n = -(-tokens // dec.block) - int(dec.held[b])
    at = (int(dec.head) + __import__("torch").arange(n)) % dec.num_blocks
    dec.block_table[b, int(dec.held[b]):int(dec.held[b]) + n] = dec.ring[at]
    dec.head += n
    dec.held[b] += n
    dec.cache_len[b] = tokens


def everyone(dec):
    import torch
    return torch.ones((dec.B,), dtype=torch.bool)


def free(dec):
    at = (__import__("torch").arange(int(dec.tail - dec.head)) + int(dec.head)) % dec.num_blocks
    return sorted(dec.ring[at].tolist())


def groups_of(dec, start, blocks):
    for b, n in zip(start, blocks):
        cached(dec, b, n * dec.block + 1)
    dec.share(start, blocks)


def test_groups_that_come_again_have_the_buffers_that_graphs_captured(ssd):
    dec = state(make(0, 0, max_blocks=9), 40)
    kept, seen = {}, 0
    for start, blocks in [([0, 2, 4], [3, 2]), ([0, 1, 2, 4], [1, 2, 0]), ([0, 3, 4], [5, 1]), ([0, 4], [2]),
                          ([0, 1, 4], [1, 3])] * 4:
        groups_of(dec, start, blocks)
        here = [t.data_ptr() for t in (dec.group_start, dec.shared)]
        assert kept.setdefault(len(blocks), here) == here
        assert dec.group_start.tolist() == start and dec.shared.tolist() == blocks
        assert dec.max_shared >= max(blocks)
        dec.release(everyone(dec))
        assert free(dec) == list(range(40))
        # nothing is kept beside the buffers of each number of groups
        assert not dec._outgrown and (seen := max(seen, len(dec._groups))) <= 3


def test_outgrown_workspaces_stay_within_twice_the_last(ssd):
    """Graphs may have captured them, so they are kept; they grow by half at least, so that however often
    a little more is needed all of them together hold at most twice what the last one does (1 / (1 - 2/3)
    less itself)."""
    ssd.ssd_set_cache_sharing(1)
    so, dec = ssd.load(), make(1, 1, B=16, max_blocks=4000)
    dec.N_max, sizes = 64, set()
    for most in list(range(1, 4000, 7)) + [5, 900, 33]:
        dec.max_shared = most
        n = dec._workspace(1)[1]
        assert n >= so.ssd_cache_attention_shared_workspace(16, 1, 8, 2, 128, 1, 64000, 16 * most)
        sizes.add(n)
        assert sum(t.numel() for t in dec._outgrown) <= 2 * n
    assert len(sizes) > 2


def test_blocks_of_a_place_that_began_anew_come_back(ssd):
    """Also those in the places of the blocks that its group shares, whichever goes first."""
    import torch
    for order in ([1, 0, 2, 3], [0, 2, 1, 3], [3, 2, 1, 0]):
        dec = state(make(0, 0, max_blocks=9), 40)
        groups_of(dec, [0, 3, 4], [4, 2])
        for b in range(3):
            cached(dec, b, 4 * 16 + 40)
        dec.release(torch.tensor([False, True, False, False]))
        assert len(free(dec)) == 40 - 4 - 3 - 3 - 3 and dec._open.tolist() == [1, -1, 1, 1]
        cached(dec, 1, 50)  # (a pass that was captured before any share())
        held = [t for t in dec.block_table.flatten().tolist() if t >= 0]
        assert len(set(held)) + len(free(dec)) == 40
        for b in order:
            dec.release(torch.arange(4) == b)
        assert free(dec) == list(range(40)) and dec.shared.tolist() == [0, 0] and dec._open.tolist() == [1] * 4


def test_share_refuses_what_would_lose_blocks(ssd):
    import torch
    dec = state(make(0, 0, max_blocks=9), 40)
    cached(dec, 0, 50)
    before = dec.block_table.clone()
    # blocks that are not cached whole, by the first of a group or at all
    for start, blocks in (([0, 4], [4]), ([0, 2, 4], [3, 1]), ([0, 1, 4], [0, 2])):
        with pytest.raises(ValueError, match="not cached"):
            dec.share(start, blocks)
    # a sequence that would join holds blocks of its own
    cached(dec, 2, 5)
    with pytest.raises(ValueError, match="holds blocks"):
        dec.share([0, 4], [3])
    assert dec.groups == 0 and torch.equal(dec.block_table[[0, 1, 3]], before[[0, 1, 3]])
    # groups that share nothing, and empty groups, may hold what they do
    dec.share([0, 2, 2, 4], [3, 1, 0])
    assert dec.block_table[1, :3].tolist() == dec.block_table[0, :3].tolist()
    # an earlier group's blocks
    with pytest.raises(ValueError, match="earlier"):
        dec.share([0, 2, 4], [3, 0])
    dec.release(torch.tensor([True, False, False, False]))
    with pytest.raises(ValueError, match="earlier"):
        dec.share([0, 4], [0])
    dec.release(everyone(dec))
    assert free(dec) == list(range(40))
    groups_of(dec, [0, 4], [2])
