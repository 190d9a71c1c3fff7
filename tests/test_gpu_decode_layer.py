"""The operators of a decoder layer together: 8-bit projections, head norms, attention over blocks
that sequences share, and the residual sum, as PagedDecode and ScaledLinear call them.

Bars.  Sequences that share blocks hold the same cached values as sequences with blocks of their own,
so only the order of sums and the rounding of probabilities differ: each call is within 4e-3 of the
2-norm (tests/test_gpu_cache_attention.py), two within 8e-3.  A layer in 8 bits against the same layer
in float64: a rounding to e4m3 is 2^-4 / sqrt 3 = 0.036 of a value in the mean of squares, so a product
of two rounded factors is off by 0.05, scores (of standard deviation about 1, of two such) by 0.07, the
cache by 0.036 twice, the values by 0.05, the way out by 0.05: 0.14 in all, and the bar is twice that;
a wrong operand gives 1."""
import os
import runpy

import numpy as np
import pytest
import torch

from oracle import cache as oc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def make(ssd, B, Hq, Hkv, d, block, prefix, W, N_max, spare=0):
    from paper_2606_20543_gb300.decode import PagedDecode
    sec = (d // 2 - 2 * (d // 8), d // 8, d // 8)
    freq = torch.from_numpy((50.0 ** -(np.arange(d // 2) / (d // 2))).astype(np.float32)).cuda()
    M = -(-(prefix + W * W) // block)
    return PagedDecode(ssd.grid(W, W, prefix), B, Hq, Hkv, d, B * M + spare, block, M, N_max, freq, sec)


def rows(gen, n, Hq, Hkv, d):
    x = torch.randn((n, (Hq + 2 * Hkv) * d), generator=gen, device="cuda").to(torch.bfloat16)
    return x.split([Hq * d, Hkv * d, Hkv * d], 1)


@pytest.fixture(autouse=True)
def sharing(ssd):
    """Also batches as small as these read shared blocks once."""
    ssd.ssd_set_cache_sharing(1)
    yield
    ssd.ssd_set_cache_sharing(0)


@pytest.mark.parametrize("Hq,Hkv,d,block,norm", [(8, 2, 128, 16, None), (4, 4, 64, 32, "rms"),
                                                 (8, 2, 128, 16, "layer")])
def test_shared_blocks_as_blocks_of_their_own(ssd, Hq, Hkv, d, block, norm):
    """The same tokens decoded with and without sharing; then every block comes back, once."""
    B, W, prefix = 7, 8, 5 * block + 7
    start, blocks = [0, 3, 3, 6, 7], [5, 0, 4, 0]
    gen = torch.Generator("cuda").manual_seed(d)
    hn = None
    if norm is not None:
        gain = torch.rand((Hq, d), generator=gen, device="cuda") + 0.5
        kg = torch.rand((Hkv, d), generator=gen, device="cuda") + 0.5
        hn = ssd.head_norm(norm, 1e-5, gain, None, kg, None)
    a, b = (make(ssd, B, Hq, Hkv, d, block, prefix, W, prefix) for _ in range(2))
    group = np.repeat(np.arange(4), np.diff(start))
    # one prompt a group
    prompts = {g: rows(gen, prefix, Hq, Hkv, d) for g in set(group.tolist())}
    q, k, v = (torch.cat([prompts[g][i] for g in group.tolist()]) for i in range(3))
    a.plan(i32([prefix] * B))
    o_a = a.attend(0, q, k, v, norm=hn).clone().view(B, prefix, -1)
    a.advance()
    first = np.array([i in start[:-1] and blocks[group[i]] > 0 for i in range(B)])
    done = np.array([blocks[g] * block for g in group])
    b.plan(i32(done * first))
    b.attend(0, q, k, v, norm=hn)
    b.advance()
    b.share(start, blocks)
    n = prefix - done
    N = int(n.max())
    part = [torch.cat([torch.cat([x.view(B, prefix, -1)[i, done[i]:],
                                  x.new_zeros((N - n[i], x.shape[1]))]) for i in range(B)]) for x in (q, k, v)]
    b.plan(i32(n), N)
    o_b = b.attend(0, *part, norm=hn).clone().view(B, N, -1)
    b.advance()
    for i in range(B):
        x, y = o_a[i, done[i]:].double(), o_b[i, :n[i]].double()
        assert (x - y).norm() <= 8e-3 * x.norm()
    for step in range(min(3 * block + 2, W * W)):
        qkv = rows(gen, B, Hq, Hkv, d)
        out = []
        for dec in (a, b):
            dec.plan(i32([1] * B), 1)
            out.append(dec.attend(0, *qkv, norm=hn).clone().double())
            dec.advance()
        assert (out[0] - out[1]).norm() <= 8e-3 * out[0].norm()
    assert int(a.status.item()) == 0 and int(b.status.item()) == 0
    assert torch.equal(a.cache_len, b.cache_len)
    free = lambda dec: int((dec.tail - dec.head).item())  # noqa: E731
    assert free(b) - free(a) == 2 * 5 + 2 * 4             # held once instead of three times
    # what a group shares goes back with its last sequence
    was = free(b)
    b.release(torch.tensor([True, True, False, False, False, False, True], device="cuda"))
    mine = -(-int(b.cache_len[2].item()) // block)
    assert free(b) == was + 2 * (mine - 5) + mine
    b.release(torch.ones((B,), dtype=torch.bool, device="cuda"))
    assert free(b) == b.num_blocks
    at = (torch.arange(b.num_blocks, device="cuda") + b.head) % b.num_blocks
    assert torch.equal(b.ring[at].sort().values, torch.arange(b.num_blocks, dtype=torch.int32, device="cuda"))
    # and the places begin anew
    b.plan(i32([prefix] * B))
    o = b.attend(0, q, k, v, norm=hn).view(B, prefix, -1).double()
    b.advance()
    assert int(b.status.item()) == 0 and (o - o_a.double()).norm() <= 8e-3 * o.norm()


def test_graphs_of_earlier_groups(ssd):
    """A pass captured before any share() attends without groups, in a workspace of its own; one
    captured after serves the next share() of as many groups."""
    B, Hq, Hkv, d, block, W, prefix = 4, 8, 2, 128, 16, 8, 1500
    gen = torch.Generator("cuda").manual_seed(3)
    a, b = (make(ssd, B, Hq, Hkv, d, block, prefix, W, prefix) for _ in range(2))
    one, qkv = i32([1] * B), [x.contiguous() for x in rows(gen, B, Hq, Hkv, d)]

    def step(dec):
        dec.plan(one, 1)
        return dec.attend(0, *qkv)

    def begin(start, blocks):
        """The same prompts in both, b's shared (start None: not)."""
        every = torch.ones((B,), dtype=torch.bool, device="cuda")
        a.release(every)
        b.release(every)
        group = np.zeros(B, int) if start is None else np.repeat(np.arange(len(blocks)), np.diff(start))
        prompts = [rows(gen, prefix, Hq, Hkv, d) for _ in range(B)]
        q, k, v = (torch.cat([prompts[g][i] for g in group]) for i in range(3))
        a.plan(i32([prefix] * B))
        a.attend(0, q, k, v)
        a.advance()
        done = np.zeros(B, int)
        if start is not None:
            done = np.array([blocks[g] * block for g in group])
            b.plan(i32(done * [int(i in start[:-1]) for i in range(B)]))
            b.attend(0, q, k, v)
            b.advance()
            b.share(start, blocks)
        n = prefix - done
        part = [torch.cat([x.view(B, prefix, -1)[i, np.r_[done[i]:prefix, 0:done[i]]] for i in range(B)])
                for x in (q, k, v)]
        b.plan(i32(n))
        b.attend(0, *part)
        b.advance()

    def capture():
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = step(b)
            b.advance()
        return graph, o

    def check(graph, o):
        for x in qkv:
            x.normal_(generator=gen)
        want = step(a).double()
        a.advance()
        graph.replay()
        torch.cuda.synchronize()
        assert (o.double() - want).norm() <= 8e-3 * want.norm()
        assert int(a.status.item()) == 0 and int(b.status.item()) == 0
        assert torch.equal(a.cache_len, b.cache_len)

    begin(None, None)
    step(b)
    size = b._ws[1][0].numel()
    assert size > 4096
    alone, o0 = capture()
    check(alone, o0)
    begin([0, 2, 4], [40, 7])
    step(b)
    shared, o1 = capture()
    junk = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for graph, o in ((shared, o1), (alone, o0), (shared, o1)):
        check(graph, o)
    assert all((t == 7).all() for t in junk)
    begin([0, 1, 4], [11, 30])
    check(shared, o1)
    check(alone, o0)
    begin([0, 4], [50])
    step(b)
    fewer, o2 = capture()
    check(fewer, o2)
    check(alone, o0)


def test_sharing_set_between_passes(ssd):
    """A pass asks for its workspace as sharing is set when it runs; a graph keeps what it was captured with."""
    B, Hq, Hkv, d, block, W, prefix = 4, 8, 2, 128, 16, 4, 1500
    gen = torch.Generator("cuda").manual_seed(9)
    dec = make(ssd, B, Hq, Hkv, d, block, prefix, W, prefix)
    dec.plan(i32([prefix, 0, 0, 0]))
    dec.attend(0, *rows(gen, B * prefix, Hq, Hkv, d))
    dec.advance()
    dec.share([0, 4], [prefix // block])
    one, qkv, out = i32([1] * B), [x.contiguous() for x in rows(gen, B, Hq, Hkv, d)], []
    for how in (2, 1, 0):
        ssd.ssd_set_cache_sharing(how)
        dec.plan(one, 1)
        out.append(dec.attend(0, *qkv).clone())
        if how == 2:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                o = dec.attend(0, *qkv)
    graph.replay()
    torch.cuda.synchronize()
    assert int(dec.status.item()) == 0 and torch.equal(o, out[0])
    for x in out[1:]:
        assert (x.double() - out[0].double()).norm() <= 4e-3 * out[0].double().norm()


def test_share_refuses(ssd):
    dec = make(ssd, 4, 2, 2, 64, 16, 40, 4, 40)
    for start, blocks in (([0, 4], []), ([0, 3], [1]), ([1, 4], [1]), ([0, 3, 2, 4], [1, 1, 1]), ([0, 4], [-1]),
                          ([0, 4], [dec.max_blocks + 1])):
        with pytest.raises(ValueError):
            dec.share(start, blocks)


@pytest.mark.parametrize("Hq,Hkv,d,norm", [(8, 2, 64, "rms"), (4, 2, 128, "layer")])
def test_a_layer_in_8_bits(ssd, Hq, Hkv, d, norm):
    """x + out(attention(norm(qkv(x)))), prompts and then tokens in a replayed graph, against float64."""
    from paper_2606_20543_gb300.scaled import ScaledLinear, ScaledRows
    B, W, prefix, block, width = 5, 4, 37, 16, Hq * d
    gen = torch.Generator("cuda").manual_seed(3)
    w1 = torch.randn(((Hq + 2 * Hkv) * d, width), generator=gen, device="cuda") * width ** -0.5
    w2 = (torch.randn((width, width), generator=gen, device="cuda") * width ** -0.5).to(torch.bfloat16)
    gain = torch.rand((d,), generator=gen, device="cuda") + 0.5
    hn = ssd.head_norm(norm, 1e-5, gain, None, gain, None)
    dec = make(ssd, B, Hq, Hkv, d, block, prefix, W, prefix)
    qkv, out, xs = ScaledLinear(w1), ScaledLinear(w2), ScaledRows(B * prefix, width)
    a, b = Hq * d, (Hq + Hkv) * d

    def layer(x):
        y = qkv(xs.quantize(x))
        return out(xs.quantize(dec.attend(0, y[:, :a], y[:, a:b], y[:, b:], norm=hn)), add=x)

    freq, sec = (50.0 ** -(np.arange(d // 2) / (d // 2))).astype(np.float32), dec.rotary.sec
    past = [np.zeros((0, 2, Hkv, d)) for _ in range(B)]
    g64, W1, W2 = gain.double().cpu().numpy(), w1.double().cpu().numpy(), w2.double().cpu().numpy()

    def reference(x, N):
        """The residual's part of every row, from the values before any rounding."""
        y = (x.double().cpu().numpy() @ W1.T).reshape(B, N, Hq + 2 * Hkv, d)
        o = np.zeros((B, N, Hq, d))
        for i in range(B):
            c = len(past[i])
            pos = np.zeros((N, 3), np.int64)
            for j in range(N):
                p = c + j
                pos[j] = p if p < prefix else (prefix, prefix + (p - prefix) // W, prefix + (p - prefix) % W)
            turn = lambda z: oc.rotate(oc.head_norm(z, norm, 1e-5, g64), pos, freq, list(sec), False)  # noqa: E731
            q, k = turn(y[i, :, :Hq]), turn(y[i, :, Hq:Hq + Hkv])
            past[i] = np.concatenate([past[i], np.stack([k, y[i, :, Hq + Hkv:]], 1)])
            see = np.arange(c + N)[None] <= c + np.arange(N)[:, None]
            o[i], *_ = oc.attention(q, past[i][:, 0], past[i][:, 1], see, d ** -0.5, np.ones((c + N, Hkv)))
        return o.reshape(B * N, Hq * d) @ W2.T

    def compare(y, x, N):
        want = reference(x, N)
        err = y.double().cpu().numpy() - x.double().cpu().numpy() - want
        assert np.linalg.norm(err) <= 0.28 * np.linalg.norm(want)

    x = torch.randn((B * prefix, width), generator=gen, device="cuda").to(torch.bfloat16)
    dec.plan(i32([prefix] * B))
    y = layer(x)
    dec.advance()
    compare(y, x, prefix)
    x, one = torch.zeros((B, width), dtype=torch.bfloat16, device="cuda"), i32([1] * B)
    y = torch.zeros_like(x)

    def step():
        dec.plan(one, 1)
        y.copy_(layer(x))
        dec.advance()

    graph = None
    for i in range(5):
        x.copy_(torch.randn((B, width), generator=gen, device="cuda"))
        if i == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is None:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        compare(y, x, 1)
    for st in (dec.status, qkv.status, out.status):
        assert int(st.item()) == 0


def test_linear_layers_shapes_and_refusals(ssd):
    from paper_2606_20543_gb300.scaled import ScaledLinear, ScaledRows
    gen = torch.Generator("cuda").manual_seed(5)
    for M, N, K in ((1, 3, 7), (9, 130, 129), (70, 64, 300)):
        w = torch.randn((N, K), generator=gen, device="cuda")
        x = torch.randn((M, 8 * (-(-K // 8)) + 8), generator=gen, device="cuda")[:, :K]
        f, r = ScaledLinear(w), ScaledRows(M + 2, K).quantize(x)
        want = x.double() @ w.double().t()
        for add in (None, torch.randn((M, N), generator=gen, device="cuda").to(torch.bfloat16)):
            y = f(r, add, dtype=torch.float32).double() - (0 if add is None else add.double())
            # factors off by 0.036 each: 0.05, twice that
            assert (y - want).norm() <= 0.1 * want.norm() + 1e-6
        buf = torch.zeros((M, 2 * N), dtype=torch.bfloat16, device="cuda")
        assert torch.equal(f(r, out=buf[:, N:]), f(r)) and (buf[:, :N] == 0).all()
        assert int(f.status.item()) == 0
    # weights that do not lie as the quantiser reads them are copied
    w = torch.randn((70, 200), generator=gen, device="cuda").to(torch.bfloat16)
    wide = torch.zeros((70, 208), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:201] = w
    for x in (wide[:, 1:201], w.t().contiguous().t(), w[:1].expand(70, 200)):
        f1, f2 = ScaledLinear(x), ScaledLinear(x.contiguous().clone())
        assert torch.equal(f1.w.view(torch.uint8), f2.w.view(torch.uint8)) and torch.equal(f1.scale, f2.scale)
    with pytest.raises(ValueError):
        ScaledRows(4, 64).quantize(torch.zeros((5, 64), device="cuda"))
    with pytest.raises(ValueError):
        ScaledRows(4, 64).quantize(torch.zeros((64, 4), device="cuda").t())
    with pytest.raises(ValueError):
        f(ScaledRows(4, 64).quantize(torch.zeros((2, 64), device="cuda")))
    with pytest.raises(ValueError):
        f(r, out=torch.zeros((M, N + 1), device="cuda"))


@pytest.mark.parametrize("argv", [["--images", "3", "--norm", "rms", "--fp8"],
                                  ["--images", "2", "--norm", "layer", "--no-graph", "--batch", "4"]])
def test_example(ssd, argv):
    """It runs, and gives tokens of the vocabulary."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    image = runpy.run_path(path)["main"](["--batch", "6", "--grid", "6", "--prefix", "40", "--vocab", "512",
                                          "--heads", "4", "2", "64", "--block", "16", "--top-k", "50"] + argv)
    assert image.shape[1] == 36 and (image >= 0).all() and (image < 512).all()
