"""The paged cache's calls together (decode.PagedDecode) against the oracle.

The attention's output is compared twice.  With the cache's own values (read back) the bounds
are those of the attention alone: bf16 of o and of a probability (2^-8 each), a score exact
to 2^-16 of its magnitude, small probabilities to 2^-16 of the largest.  With the keys and
values before they were cached, e4m3's rounding comes on top: at most 2^-4 of an entry,
2^-4 / sqrt 3 = 0.036 in the mean, once in V and, as an absolute error of scores of standard
deviation 1, once in K; entries that a growing scale rounds again carry it up to three times.
0.036 * sqrt(2 * 3) = 0.09 of the 2-norm; the bar is twice that, and a key or a value out of its
place gives 1."""
import os
import runpy

import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import sample as os_

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


class Shadow:
    """What the oracle knows of the same batch: every sequence's rotated keys and values."""

    def __init__(self, dec, freq, sections, interleaved):
        self.dec, self.freq, self.sec, self.inter = dec, freq, sections, interleaved
        self.k = [np.zeros((0, dec.Hkv, dec.d)) for _ in range(dec.B)]
        self.v = [np.zeros((0, dec.Hkv, dec.d)) for _ in range(dec.B)]

    def positions(self, first, n):
        g = self.dec.g
        out = np.zeros((n, 3), np.int64)
        for j in range(n):
            p = first + j
            if p < g.prefix_len:
                out[j] = p
            else:
                y, x = divmod(p - g.prefix_len, g.row_stride)
                out[j] = g.prefix_len, g.prefix_len + y, g.prefix_len + x
        return out

    def cached(self, b, L):
        """The cache's values of sequence b, and V's scales, as the device holds them."""
        dec = self.dec
        t = dec.block_table[b].cpu().numpy()
        out = []
        for x, s in ((dec.k[0], dec.k_scale[0]), (dec.v[0], dec.v_scale[0])):
            ids = t[np.arange(L) // dec.block]
            code = x.view(torch.uint8).cpu().numpy()[ids, :, np.arange(L) % dec.block]
            scale = s.cpu().numpy().astype(np.float64)[ids]
            out += [oc.TABLE[code] * scale[:, :, None], scale]
        return out[0], out[2], out[3]

    def one_pass(self, new, N, rng, draft_pos=None):
        dec = self.dec
        B, Hq, Hkv, d = dec.B, dec.Hq, dec.Hkv, dec.d
        cache = dec.cache_len.cpu().numpy()
        qkv = torch.from_numpy(rng.standard_normal((B * N, (Hq + 2 * Hkv) * d)).astype(np.float32))
        qkv = qkv.to(torch.bfloat16).cuda()
        a, b_ = Hq * d, (Hq + Hkv) * d
        dec.plan(i32(new), N)
        o = dec.attend(0, qkv[:, :a], qkv[:, a:b_], qkv[:, b_:],
                       None if draft_pos is None else i32(draft_pos))
        assert int(dec.status.item()) == 0
        o = o.double().cpu().numpy().reshape(B, N, Hq, d)
        x = qkv.double().cpu().numpy().reshape(B, N, Hq + 2 * Hkv, d)
        g = dec.g
        num = den = 0.0
        for b in range(B):
            n, c = int(new[b]), int(cache[b])
            if n == 0:
                continue
            pos = self.positions(c, n)
            q = oc.rotate(x[b, :n, :Hq], pos, self.freq, self.sec, self.inter)
            k = oc.rotate(x[b, :n, Hq:Hq + Hkv], pos, self.freq, self.sec, self.inter)
            self.k[b] = np.concatenate([self.k[b][:c], k])
            self.v[b] = np.concatenate([self.v[b][:c], x[b, :n, Hq + Hkv:]])
            kp, qp = np.arange(c + n), c + np.arange(n)
            if draft_pos is not None:
                i = np.asarray(draft_pos[b])[:n]
                qp = g.prefix_len + i // g.grid_w * g.row_stride + i % g.grid_w
                kp = np.concatenate([kp[:c], qp])
            see = kp[None] <= qp[:, None]
            ck, cv, cs = self.cached(b, c + n)
            q16 = torch.from_numpy(q).to(torch.bfloat16).double().numpy()
            ref, _, A, F, mag = oc.attention(q16, ck, cv, see, d ** -0.5, cs)
            # (the device rounds its rotated q to bf16 from float32: an ulp apart at times)
            off = (2.0 ** -16 * mag + 2.0 ** -8 * mag)[..., None]
            tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * off) * A + 2.0 ** -16 * F + 1e-30
            assert np.all(np.abs(o[b, :n] - ref) <= tol)
            full, *_ = oc.attention(q, self.k[b], self.v[b], see, d ** -0.5, np.ones((c + n, Hkv)))
            num += np.sum((o[b, :n] - full) ** 2)
            den += np.sum(full ** 2)
        assert num <= 0.18 ** 2 * den


@pytest.mark.parametrize("Hq,Hkv,d,block,interleaved", [(4, 2, 64, 16, False), (8, 1, 128, 32, True),
                                                        (2, 2, 128, 16, False)])
def test_prompts_tokens_drafts_and_reuse(ssd, Hq, Hkv, d, block, interleaved):
    from paper_2606_20543_gb300.decode import PagedDecode
    rng = np.random.default_rng(Hq * d + block)
    B, H, W, prefix = 3, 5, 6, 21
    sec = (d // 2 - 2 * (d // 8), d // 8, d // 8)
    freq = (50.0 ** -(np.arange(d // 2) / (d // 2))).astype(np.float32)
    M = -(-(prefix + H * W) // block)
    dec = PagedDecode(ssd.grid(H, W, prefix), B, Hq, Hkv, d, B * M, block, M, 40,
                      torch.from_numpy(freq).cuda(), sec, interleaved)
    dec.k.view(torch.uint8).fill_(0x7f)  # NaN wherever nothing was written
    dec.v.view(torch.uint8).fill_(0x7f)
    sh = Shadow(dec, freq, sec, interleaved)
    sh.one_pass([21, 21, 21], 40, rng)  # prompts
    dec.advance()
    for _ in range(4):  # one token each
        sh.one_pass([1, 1, 1], 1, rng)
        dec.advance()
    # drafts: the rest of row 0 and the row below, of which some stay
    at = int(dec.cache_len[0].item()) - prefix
    drafts = np.arange(at, 2 * W)
    pos = np.tile(drafts, (B, 1))
    sh.one_pass([len(drafts)] * B, len(drafts), rng, pos)
    dec.advance(i32([len(drafts), 2, 0]))
    sh.one_pass([1, 1, 1], 1, rng)
    dec.advance()
    # sequence 1 ends; its blocks serve its next image, among them in another order
    held = dec.held.clone()
    tail = int(dec.tail.item())
    dec.release(torch.tensor([False, True, False], device="cuda"))
    assert int(dec.tail.item()) == tail + int(held[1].item())
    sh.one_pass([1, 30, 0], 30, rng)
    dec.advance()
    free = int((dec.tail - dec.head).item())
    ids = [int(x) for x in dec.ring[:-1].roll(-int(dec.head.item()) % dec.num_blocks)[:free]]
    for b in range(B):
        ids += [int(x) for x in dec.block_table[b, :int(dec.held[b].item())]]
    assert sorted(ids) == list(range(dec.num_blocks))  # every block is free or held, once


def test_sampling_through_the_batch(ssd):
    from paper_2606_20543_gb300.decode import PagedDecode
    rng = np.random.default_rng(5)
    B, V = 4, 1000
    dec = PagedDecode(ssd.grid(4, 4, 0), B, 1, 1, 64, 8, 16, 2, 1, torch.ones(32, device="cuda"),
                      (32, 0, 0))
    x = torch.from_numpy((2 * rng.standard_normal((B, V))).astype(np.float32)).cuda()
    u = torch.from_numpy(rng.random((B, 2)).astype(np.float32)).cuda()
    tok = dec.sample(x, ssd.sampling(0.9, 50, 0.8), ssd.rng(uniforms=u)).cpu().numpy()
    assert int(dec.status.item()) == 0
    for r in range(B):
        ref = os_.sample_row(x[r].cpu().numpy(), 0.9, 50, 0.8, 0.0, float(u[r, 1]))
        assert tok[r] in ref["ids"]
        assert ref["lo"] <= int(dec.kept[r].item()) <= ref["hi"]


def test_refusals(ssd):
    from paper_2606_20543_gb300.decode import PagedDecode
    dec = PagedDecode(ssd.grid(4, 4, 0), 2, 2, 1, 64, 8, 16, 2, 3, torch.ones(32, device="cuda"),
                      (32, 0, 0))
    with pytest.raises(ValueError):
        dec.plan(i32([1, 1]), 4)
    dec.plan(i32([1, 1]), 1)
    q = torch.zeros((2, 128), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in ((q.float(), k, k), (q, q, k), (q[:1], k, k)):
        with pytest.raises(ValueError):
            dec.attend(0, *bad)
    with pytest.raises(ValueError):
        dec.sample(torch.zeros((7, 10), device="cuda"), ssd.sampling(), ssd.rng())


def test_example_with_and_without_a_graph(ssd):
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "paged_decode.py")
    main = runpy.run_path(path)["main"]
    args = ["--batch", "2", "--grid", "6", "--prefix", "9", "--vocab", "500", "--heads", "4", "2",
            "64", "--block", "16", "--top-k", "100"]
    with_graph = main(args)
    assert with_graph.shape == (2, 36)
    assert bool(((with_graph >= 0) & (with_graph < 500)).all())
    assert torch.equal(with_graph, main(args + ["--no-graph"]))
