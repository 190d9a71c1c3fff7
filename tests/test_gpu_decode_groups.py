"""PagedDecode.share() again and again: graphs of earlier numbers of groups, places that are released
while their group goes on, and calls that it refuses.  Bars as in tests/test_gpu_decode_layer.py: the
shared and the unshared attention hold the same cached values, so a call is within 4e-3 of the 2-norm,
two within 8e-3."""
import numpy as np
import pytest
import torch

from tests.test_gpu_decode_layer import i32, make, rows

pytestmark = pytest.mark.gpu

B, HQ, HKV, D, BLOCK, W, PREFIX = 4, 8, 2, 128, 16, 8, 700


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


@pytest.fixture(autouse=True)
def sharing(ssd):
    ssd.ssd_set_cache_sharing(1)
    yield
    ssd.ssd_set_cache_sharing(0)


class Pair:
    """The same tokens in a decoder without sharing (a) and one with (b)."""

    def __init__(self, ssd, seed):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.a, self.b = (make(ssd, B, HQ, HKV, D, BLOCK, PREFIX, W, PREFIX) for _ in range(2))
        self.one = i32([1] * B)
        self.qkv = [x.contiguous() for x in rows(self.gen, B, HQ, HKV, D)]

    def begin(self, start, blocks):
        a, b = self.a, self.b
        every = torch.ones((B,), dtype=torch.bool, device="cuda")
        a.release(every)
        b.release(every)
        group = np.repeat(np.arange(len(blocks)), np.diff(start))
        prompts = [rows(self.gen, PREFIX, HQ, HKV, D) for _ in blocks]
        q, k, v = (torch.cat([prompts[g][i] for g in group]) for i in range(3))
        a.plan(i32([PREFIX] * B))
        a.attend(0, q, k, v)
        a.advance()
        done = np.array([blocks[g] * BLOCK for g in group])
        b.plan(i32(done * [int(i in start[:-1]) for i in range(B)]))
        b.attend(0, q, k, v)
        b.advance()
        b.share(start, blocks)
        b.plan(i32(PREFIX - done))
        b.attend(0, *[torch.cat([x.view(B, PREFIX, -1)[i, np.r_[done[i]:PREFIX, 0:done[i]]] for i in range(B)])
                      for x in (q, k, v)])
        b.advance()

    def step(self, dec, n=None):
        dec.plan(self.one if n is None else n, 1)
        return dec.attend(0, *self.qkv)

    def capture(self):
        self.step(self.b)  # (its workspace)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = self.step(self.b)
            self.b.advance()
        return graph, o

    def check(self, graph, o):
        for x in self.qkv:
            x.normal_(generator=self.gen)
        want = self.step(self.a).double()
        self.a.advance()
        o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert (o.double() - want).norm() <= 8e-3 * want.norm()
        assert int(self.a.status.item()) == 0 and int(self.b.status.item()) == 0
        assert torch.equal(self.a.cache_len, self.b.cache_len)


def test_graphs_of_as_many_groups_serve_later_groups(ssd):
    p = Pair(ssd, 3)
    p.begin([0, 2, 4], [40, 7])
    two = p.capture()
    p.check(*two)
    p.begin([0, 1, 3, 4], [12, 30, 5])
    three = p.capture()
    p.check(*three)
    p.begin([0, 3, 4], [9, 33])      # two again
    p.check(*two)
    p.begin([0, 2, 2, 4], [20, 1, 25])
    p.check(*three)
    p.begin([0, 1, 4], [43, 43])     # more blocks than the graph was captured with: captured anew
    more = p.capture()
    p.check(*more)
    p.begin([0, 2, 4], [3, 40])
    p.check(*two)
    p.check(*more)


@pytest.mark.parametrize("captured", [False, True])
def test_a_place_whose_group_goes_on_without_it(ssd, captured):
    """A pass that asks tokens of it leaves it out and says so; the others' rows are right, and the place
    begins anew when its group is done."""
    p = Pair(ssd, 7)
    p.begin([0, 3, 4], [20, 31])
    graph = p.capture() if captured else None
    gone = torch.tensor([False, True, False, False], device="cuda")
    p.a.release(gone)
    p.b.release(gone)
    held = int((p.b.tail - p.b.head).item())
    # without tokens for it nothing is wrong; with them (or fewer than none) it is left out
    for n in (0, 1, -1):
        want = p.step(p.a, i32([1, 0, 1, 1])).clone().double()
        p.a.advance()
        p.b._o.fill_(5.0)
        if captured and n == 1:
            graph[0].replay()
            o = graph[1]
        else:
            o = p.step(p.b, i32([1, n, 1, 1]))
            p.b.advance()
        torch.cuda.synchronize()
        assert int(p.b.status.item()) == (0 if n == 0 else 6) and int(p.a.status.item()) == 0
        p.b.status.zero_()
        keep = [0, 2, 3]
        assert (o[keep].double() - want[keep]).norm() <= 8e-3 * want[keep].norm() and (o[1] == 5.0).all()
        assert p.b.n_new.tolist() == [1, 0, 1, 1] and p.b.cache_len.tolist() == p.a.cache_len.tolist()
        assert int(p.b.held[1].item()) == 0
    assert held - int((p.b.tail - p.b.head).item()) <= 3  # (blocks that the three others went on into)
    for b in (2, 0, 3):
        p.b.release(torch.arange(B, device="cuda") == b)
    assert int((p.b.tail - p.b.head).item()) == p.b.num_blocks
    at = (torch.arange(p.b.num_blocks, device="cuda") + p.b.head) % p.b.num_blocks
    assert torch.equal(p.b.ring[at].sort().values, torch.arange(p.b.num_blocks, dtype=torch.int32, device="cuda"))
    p.begin([0, 2, 4], [11, 17])
    p.check(*p.capture())


def test_a_place_that_began_anew_without_groups(ssd):
    """A graph of before any share() serves it; a pass with groups leaves it out until its group is done."""
    p = Pair(ssd, 8)
    alone = p.capture()
    p.b.release(torch.ones((B,), dtype=torch.bool, device="cuda"))
    p.begin([0, 4], [9])
    gone = torch.tensor([False, False, True, False], device="cuda")
    p.a.release(gone)
    p.b.release(gone)
    for _ in range(3):
        p.check(*alone)
    p.step(p.b)
    torch.cuda.synchronize()
    assert int(p.b.status.item()) == 6 and p.b.n_new.tolist() == [1, 1, 0, 1]
    p.b.status.zero_()
    rest = torch.tensor([True, True, False, True], device="cuda")
    p.a.release(rest)
    p.b.release(rest)
    want = p.step(p.a).clone().double()
    o = p.step(p.b)
    torch.cuda.synchronize()
    assert int(p.b.status.item()) == 0 and (o.double() - want).norm() <= 8e-3 * want.norm()
    p.b.release(torch.ones((B,), dtype=torch.bool, device="cuda"))
