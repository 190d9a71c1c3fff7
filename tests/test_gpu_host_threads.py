"""Calls of one operator from two host threads, each on a stream of its own, with sizes that need
different amounts of shared memory: every call is accepted and gives what it gives alone.  (The
limit of a kernel's shared memory belongs to the process: a call that sets it to its own need
takes it from the other thread's launch.)"""
import threading

import pytest
import torch

from tests.test_gpu_cache_attention import i32, ssd  # noqa: F401

pytestmark = pytest.mark.gpu

CALLS = 4000


def together(calls, outputs):
    """calls: one function (stream) per thread; outputs: the tensors that each writes."""
    streams = [torch.cuda.Stream() for _ in calls]
    alone = []
    for call, stream, out in zip(calls, streams, outputs):
        call(stream)
        torch.cuda.synchronize()
        alone.append([x.clone() for x in out])
        for x in out:
            x.zero_()
    torch.cuda.synchronize()
    gate, errors = threading.Barrier(len(calls)), []

    def work(call, stream):
        gate.wait()
        try:
            for _ in range(CALLS):
                call(stream)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=x) for x in zip(calls, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for out, ref in zip(outputs, alone):
        for x, y in zip(out, ref):
            assert torch.equal(x, y)


def test_sampler(ssd):  # noqa: F811
    gen = torch.Generator("cuda").manual_seed(1)
    calls, outputs = [], []
    for V in (300, 200000):
        x = torch.randn((1, V), generator=gen, device="cuda")
        u = torch.rand((1, 2), generator=gen, device="cuda")
        tok, st = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        p, r = ssd.sampling(1.0, 50, 0.9), ssd.rng(uniforms=u)

        def call(stream, x=x, u=u, V=V, p=p, r=r, tok=tok, st=st):
            ssd.ssd_sample(1, V, x, V, p, r, tok, None, None, st, stream=stream)
        calls.append(call)
        outputs.append([tok, st])
    together(calls, outputs)


@pytest.mark.parametrize("D,Hq,tokens", [(1, 4, (64, 160000)), (3, 4, (80000, 320000)),
                                         (24, 2, (80000, 800000))])
def test_cache_attention(ssd, D, Hq, tokens):  # noqa: F811
    """The 8-row, 16-row and tensor-core kernels, under tables of two widths."""
    gen = torch.Generator("cuda").manual_seed(D)
    Hkv, d, block, cache = 1, 128, 16, 40
    pool = -(-(cache + D) // block)

    def new(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    k, v = (new(pool, Hkv, block, d).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.ones((pool, Hkv), device="cuda") for _ in range(2))
    c, g = ssd.cache(k, v, ks, vs), ssd.grid(16, 16, 0)
    calls, outputs = [], []
    for L in tokens:
        M = L // block
        table = torch.full((1, M), -1, dtype=torch.int32, device="cuda")
        table[0, :pool] = torch.arange(pool, device="cuda")
        q = new(1, D, Hq, d).to(torch.bfloat16)
        o, st = torch.zeros_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
        n = ssd.ssd_cache_attention_workspace(1, Hq, Hkv, d, D, L)
        ws = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")
        cl, nd = i32([cache]), i32([D])

        def call(stream, M=M, table=table, q=q, o=o, st=st, n=n, ws=ws, cl=cl, nd=nd):
            ssd.ssd_cache_attention(g, c, 1, Hq, cl, nd, None, None, D, table, M, q, 0.0, o, None, ws, n,
                                    st, stream=stream)
        calls.append(call)
        outputs.append([o, st])
    together(calls, outputs)


def test_acceptance(ssd):  # noqa: F811
    gen = torch.Generator("cuda").manual_seed(2)
    calls, outputs = [], []
    for V in (256, 131072):
        t, r = (torch.randn((1, V), generator=gen, device="cuda") for _ in range(2))
        u = torch.rand((1, 2), generator=gen, device="cuda")
        tok, st = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        acc = torch.zeros(1, dtype=torch.uint8, device="cuda")
        rng = ssd.rng(uniforms=u)

        def call(stream, V=V, t=t, r=r, u=u, rng=rng, tok=tok, acc=acc, st=st):
            ssd.ssd_accept(1, V, t, r, V, None, 1.0, rng, tok, acc, None, None, st, stream=stream)
        calls.append(call)
        outputs.append([tok, acc, st])
    together(calls, outputs)
