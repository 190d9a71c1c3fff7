"""ssd_cache_attention_shared on two streams at once, every call into buffers of its own, and while
another thread sets the sharing switch."""
import threading

import pytest
import torch

from tests.test_gpu_cache_shared import Batch

pytestmark = pytest.mark.gpu

O, LSE, WS, BYTES, STATUS = 17, 18, 19, 20, 21  # among the call's arguments


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


def batch(seed, n, D, Hq, Hkv):
    return Batch(seed=seed, start=[0, n // 3, n], shared=[30, 60], own=[20 + 31 * i % 400 for i in range(n)],
                 nd=[D] * n, D=D, Hq=Hq, Hkv=Hkv, d=128, block=16)


@pytest.mark.parametrize("D,Hq,Hkv", [(1, 8, 2), (1, 4, 4), (40, 4, 2)])
def test_every_call_of_two_streams(ssd, D, Hq, Hkv):
    rounds, calls = 12, []
    for seed, n in ((1, 6), (2, 40)):
        b = batch(seed, n, D, Hq, Hkv)
        o, ls, st = b.run(ssd)
        assert st == 0 and b.shares
        outs = [(torch.full_like(o, 7.0), torch.full_like(ls, 7.0)) for _ in range(rounds)]
        calls.append((b, o.clone(), ls.clone(), outs, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for r in range(rounds):
        for b, _, _, outs, stream in calls:
            args = list(b.args)
            args[O], args[LSE] = outs[r]
            ssd.ssd_cache_attention_shared(*args, stream=stream)
    torch.cuda.synchronize()
    for b, o, ls, outs, _ in calls:
        assert b.args[STATUS].item() == 0
        for x, y in outs:
            assert torch.equal(x.view(torch.int16), o.view(torch.int16)) and torch.equal(y, ls)


def test_the_switch_set_by_another_thread(ssd):
    """A call goes the way its workspace suffices for, or is refused; nothing is written behind it."""
    b = batch(3, 40, 1, 8, 2)
    o, _, st = b.run(ssd)
    assert st == 0 and b.shares
    need, want = {}, {}
    for how in (1, 2):
        ssd.ssd_set_cache_sharing(how)
        need[how] = ssd.ssd_cache_attention_shared_workspace(b.B, b.groups, b.Hq, b.Hkv, b.d, b.D, b.M * b.block,
                                                             b.max_shared * b.block)
        ssd.ssd_cache_attention_shared(*b.args)
        torch.cuda.synchronize()
        want[how] = o.clone()
    small, large = sorted(need.values())
    assert small < large
    ws = torch.full((large + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    stop = threading.Event()

    def toggle():
        how = 1
        while not stop.is_set():
            how = 3 - how
            ssd.load().ssd_set_cache_sharing(how)

    other = threading.Thread(target=toggle)
    other.start()
    done = refused = 0
    try:
        for i in range(4000):
            args = list(b.args)
            args[WS], args[BYTES] = ws, small
            o.fill_(7.0)
            try:
                ssd.ssd_cache_attention_shared(*args)
            except ssd.SsdError:
                refused += 1
                continue
            done += 1
            if i % 8 == 0:
                torch.cuda.synchronize()
                assert any(torch.equal(o.view(torch.int16), w.view(torch.int16)) for w in want.values())
    finally:
        stop.set()
        other.join()
    torch.cuda.synchronize()
    assert done > 0 and b.args[STATUS].item() == 0
    assert (ws[small:] == 0xa5).all()
