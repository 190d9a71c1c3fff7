"""PagedDecode with drafts that are not the next tokens of the flat sequence, and with a pool that
cannot serve everyone.

The rotated query and the cached entries are compared with float64 rotations by the drafts' own
grid positions: bf16's rounding (2^-8 of the value) and e4m3's (half a step times the scale), each
with the float32 rotation's 2^-22 of the pair's magnitude on top.  The attention is compared over what the device
holds (its rotated q, its cache), with the bounds of test_gpu_cache_attention."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.test_gpu_cache_attention import i32, ssd  # noqa: F401

pytestmark = pytest.mark.gpu

H, W, PREFIX = 6, 7, 10
SSD_ERR_WORKSPACE = 7


class Batch:
    def __init__(self, ssd, B, Hq, Hkv, d, block, row_stride, num_blocks, N, interleaved=False):  # noqa: F811
        from paper_2606_20543_gb300.decode import PagedDecode
        self.ssd, self.rs, self.inter = ssd, row_stride, interleaved
        self.sec = (d // 2 - 2 * (d // 8), d // 8, d // 8)
        self.freq = (50.0 ** -(np.arange(d // 2) / (d // 2))).astype(np.float32)
        M = -(-(PREFIX + H * row_stride) // block)
        self.dec = PagedDecode(ssd.grid(H, W, PREFIX, row_stride), B, Hq, Hkv, d, num_blocks or B * M,
                               block, M, N, torch.from_numpy(self.freq).cuda(), self.sec, interleaved)
        self.rng = np.random.default_rng(d + block + row_stride)

    def flat_axes(self, p):
        p = np.asarray(p)
        y, x = np.divmod(p - PREFIX, self.rs)
        at = np.stack([np.full_like(p, PREFIX), PREFIX + y, PREFIX + x], -1)
        return np.where((p < PREFIX)[:, None], p[:, None], at)

    def one_pass(self, new, N, draft_pos=None, served=None):
        """One pass over all sequences; those not `served` are left out.  Returns o."""
        dec = self.dec
        B, Hq, Hkv, d = dec.B, dec.Hq, dec.Hkv, dec.d
        served = [True] * B if served is None else served
        cache = dec.cache_len.cpu().numpy()
        x = self.rng.standard_normal((B * N, (Hq + 2 * Hkv) * d)).astype(np.float32)
        x = torch.from_numpy(x).to(torch.bfloat16).cuda()
        a, b_ = Hq * d, (Hq + Hkv) * d
        dec._o.fill_(7.0)
        dec._q.fill_(7.0)
        dec.plan(i32(new), N)
        o = dec.attend(0, x[:, :a], x[:, a:b_], x[:, b_:],
                       None if draft_pos is None else i32(draft_pos))
        o = o.double().cpu().numpy().reshape(B, N, Hq, d)
        q_dev = dec._q[:B * N * a].double().cpu().numpy().reshape(B, N, Hq, d)
        x = x.double().cpu().numpy().reshape(B, N, Hq + 2 * Hkv, d)
        table = dec.block_table.cpu().numpy()
        for b in range(B):
            n, c = int(new[b]) if served[b] else 0, int(cache[b])
            assert np.all(o[b, n:] == 7.0) and np.all(q_dev[b, n:] == 7.0)
            if n == 0:
                continue
            qp = c + np.arange(n)
            if draft_pos is not None:
                i = np.asarray(draft_pos[b])[:n]
                qp = PREFIX + i // W * self.rs + i % W
            kp = np.concatenate([np.arange(c), qp])
            pos = self.flat_axes(qp)
            q, k = (oc.rotate(x[b, :n, s], pos, self.freq, self.sec, self.inter)
                    for s in (slice(0, Hq), slice(Hq, Hq + Hkv)))
            big = np.abs(x[b, :n]).max(-1, keepdims=True)
            assert np.all(np.abs(q_dev[b, :n] - q) <= 2.0 ** -8 * np.abs(q) + 2.0 ** -22 * big[:, :Hq])
            kc, vc, ks, vs = self.cached(b, c + n, table)
            for got, want, s in ((kc, k, ks), (vc, x[b, :n, Hq + Hkv:], vs)):
                got, s = got[c:], s[c:, :, None]
                # (an entry that a later token's scale rounded again is off by a second half step)
                step = oc.e4m3_step(np.maximum(np.abs(want), np.abs(got)) / s) * s
                assert np.all(np.abs(got - want) <= 0.5 * step * (1 + 2.0 ** -20) + 2.0 ** -22 * big.max())
            see = kp[None] <= qp[:, None]
            ref, _, A, F, mag = oc.attention(q_dev[b, :n], kc, vc, see, d ** -0.5, vs)
            off = (2.0 ** -16 * mag)[..., None]
            tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * off) * A + 2.0 ** -16 * F + 1e-30
            assert np.all(np.abs(o[b, :n] - ref) <= tol)
        return o

    def cached(self, b, L, table):
        dec = self.dec
        ids, at = table[b][np.arange(L) // dec.block], np.arange(L) % dec.block
        out = []
        for x, s in ((dec.k[0], dec.k_scale[0]), (dec.v[0], dec.v_scale[0])):
            code = x.view(torch.uint8).cpu().numpy()[ids, :, at]
            scale = s.cpu().numpy().astype(np.float64)[ids]
            out += [oc.TABLE[code] * scale[:, :, None], scale]
        return out[0], out[2], out[1], out[3]


@pytest.mark.parametrize("row_stride", [W, W + 1])
@pytest.mark.parametrize("Hq,Hkv,d,interleaved", [(4, 2, 64, True), (2, 2, 128, False)])
def test_drafts_turn_by_their_own_positions(ssd, row_stride, Hq, Hkv, d, interleaved):  # noqa: F811
    """Across a row's end, out of order, and with gaps."""
    t = Batch(ssd, 3, Hq, Hkv, d, 16, row_stride, 0, 16, interleaved)
    dec = t.dec
    t.one_pass([PREFIX] * 3, PREFIX)
    dec.advance()
    drafts = np.stack([np.arange(2 * W), t.rng.permutation(2 * W), 1 + 2 * np.arange(2 * W)])
    t.one_pass([2 * W, 2 * W, 2 * W - 3], 2 * W, drafts)
    assert int(dec.status.item()) == 0
    # the draft positions are a pass's, not the next one's
    dec.advance(i32([0, 0, 0]))
    t.one_pass([1, 2, 0], 2)
    assert int(dec.status.item()) == 0


def test_a_draft_outside_the_grid_is_recorded(ssd):  # noqa: F811
    t = Batch(ssd, 1, 2, 1, 64, 16, W, 0, 10)
    t.one_pass([PREFIX], PREFIX)
    t.dec.advance()
    for bad in (-1, H * W, 2 ** 30):
        t.dec.status.zero_()
        t.dec.plan(i32([2]), 2)
        z = torch.zeros((2, 2 * 64), dtype=torch.bfloat16, device="cuda")
        t.dec.attend(0, z, z[:, :64], z[:, :64], i32([[0, bad]]))
        assert int(t.dec.status.item()) == 6


def test_the_frontier_s_drafts(ssd):  # noqa: F811
    """Drafts as ssd_frontier gives them, padding slots -1, at two places of the grid."""
    t = Batch(ssd, 2, 2, 2, 64, 16, W, 0, 2 * W)
    dec = t.dec
    t.one_pass([PREFIX, PREFIX + 4], 2 * W)
    dec.advance()
    nd, pos = torch.zeros(2, dtype=torch.int32, device="cuda"), \
        torch.zeros((2, 2 * W), dtype=torch.int32, device="cuda")
    ssd.ssd_frontier(dec.g, 2, dec.cache_len, 2 * W, nd, pos, dec.status)
    t.one_pass(nd.tolist(), 2 * W, pos.tolist())
    assert nd.tolist() == [2 * W, 2 * W - 4] and int(dec.status.item()) == 0


def test_a_pool_that_runs_dry(ssd):  # noqa: F811
    """The sequence that gets no blocks is left out of the pass and does not advance, whatever
    advance() is told; once blocks are back it is served like any other."""
    t = Batch(ssd, 3, 4, 2, 64, 16, W, 5, 32)
    dec = t.dec
    dec.k.view(torch.uint8).fill_(0x7f)
    dec.v.view(torch.uint8).fill_(0x7f)
    t.one_pass([32, 20, 17], 32, served=[True, True, False])
    assert int(dec.status.item()) == SSD_ERR_WORKSPACE
    dec.advance()
    assert dec.cache_len.tolist() == [32, 20, 0] and dec.held.tolist() == [2, 2, 0]
    # one block is left: the next to ask takes it, the one behind it waits
    dec.status.zero_()
    t.one_pass([1, 1, 1], 1, served=[True, True, False])
    assert int(dec.status.item()) == SSD_ERR_WORKSPACE
    dec.advance(i32([1, 0, 1]))
    assert dec.cache_len.tolist() == [33, 20, 0] and dec.held.tolist() == [3, 2, 0]
    # sequence 0 ends; sequence 2 takes its blocks
    dec.release(torch.tensor([True, False, False], device="cuda"))
    dec.status.zero_()
    assert dec.block_table[0].tolist() == [-1] * dec.max_blocks
    t.one_pass([0, 3, 25], 25)
    dec.advance()
    assert int(dec.status.item()) == 0
    assert dec.cache_len.tolist() == [0, 23, 25] and dec.held.tolist() == [0, 2, 2]
    # and a sequence that was released and is not served holds nothing of another's
    dec.status.zero_()
    t.one_pass([17, 1, 1], 17, served=[False, True, True])
    assert int(dec.status.item()) == SSD_ERR_WORKSPACE
    dec.advance()
    assert dec.cache_len.tolist() == [0, 24, 26]


def test_more_tokens_than_a_sequence_has_room_for(ssd):  # noqa: F811
    """Lengths beyond the table are recorded, and that sequence is left out in the same way."""
    t = Batch(ssd, 2, 2, 1, 64, 16, W, 0, 16)
    dec = t.dec
    room = dec.max_blocks * dec.block
    dec.cache_len.copy_(i32([room - 3, 0]))
    dec.held.copy_(i32([dec.max_blocks, 0]))
    dec.block_table[0] = torch.arange(dec.max_blocks, dtype=torch.int32, device="cuda")
    dec.head.fill_(dec.max_blocks)
    t.one_pass([4, 5], 16, served=[False, True])
    assert int(dec.status.item()) == 6
    dec.advance()
    assert dec.cache_len.tolist() == [room - 3, 5]


def test_a_dry_pool_in_a_graph(ssd):  # noqa: F811
    """Nobody can look between the passes of a captured graph: a token each until the pool is
    empty, and two more."""
    t = Batch(ssd, 2, 2, 1, 64, 16, W, 3, 1)
    dec = t.dec
    x = torch.randn((2, 4 * 64), device="cuda").to(torch.bfloat16)
    one = i32([1, 1])

    def step():
        dec.plan(one, 1)
        dec.attend(0, x[:, :128], x[:, 128:192], x[:, 192:])
        dec.advance()

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(15):
        graph.replay()
    torch.cuda.synchronize()
    assert int(dec.status.item()) == 0 and dec.cache_len.tolist() == [16, 16]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(dec.status.item()) == SSD_ERR_WORKSPACE
    assert dec.cache_len.tolist() == [19, 16] and dec.held.tolist() == [2, 1]


def test_one_row_with_any_stride(ssd):  # noqa: F811
    """A tensor of one row may have any row stride: one new token of one sequence."""
    def one(width, stride):
        x = torch.randn(width, generator=torch.Generator("cuda").manual_seed(width), device="cuda")
        return x.to(torch.bfloat16).as_strided((1, width), (stride, 1))

    out = []
    for stride in (4096, 1, 0):
        dec = Batch(ssd, 1, 2, 1, 64, 16, W, 0, 1).dec
        dec.plan(i32([1]), 1)
        o = dec.attend(0, one(128, stride), one(64, stride), one(64, stride)).clone()
        x = one(100, stride)
        tok = dec.sample(x, ssd.sampling(1.0, 10), ssd.rng(3, 4)).clone()
        assert int(dec.status.item()) == 0
        out.append((o, tok))
    for o, tok in out[1:]:
        assert torch.equal(o, out[0][0]) and torch.equal(tok, out[0][1])


def test_refused_positions_and_starts(ssd):  # noqa: F811
    dec = Batch(ssd, 2, 2, 1, 64, 16, W, 0, 4).dec
    dec.plan(i32([1, 1]), 2)
    q = torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    pos, start = i32([[0, 1], [0, 1]]), i32([0, 0])
    for bad in (pos.long(), pos[:1], pos.t(), pos.float()):
        with pytest.raises(ValueError):
            dec.attend(0, q, k, k, bad)
    for bad in (start.long(), start[:1], i32([0, 0, 0, 0])[::2]):
        with pytest.raises(ValueError):
            dec.attend(0, q, k, k, key_start=bad)
    dec.attend(0, q, k, k, pos, start)
    assert int(dec.status.item()) == 0
