"""ssd_cache_attention on the kernels and cuts that small calls do not take: tables for long
sequences (which say how much work a call may hold), and more sequences than come out even
on the GPU's CTAs.  Tolerances as in test_gpu_cache_attention."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache_attention import attend, check, i32, ssd  # noqa: F401

pytestmark = pytest.mark.gpu

WIDE = 40960  # tokens of a table


@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("D", [17, 40, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 64), (6, 2, 64), (2, 2, 128), (8, 2, 128)])
def test_drafts_of_every_count_under_wide_tables(ssd, D, Hq, Hkv, d, block):  # noqa: F811
    cache = [70, 0, 333, 9]
    nd = [D, max(1, D - 1), D // 2, 0]
    o, ls, st, refs = attend(ssd, seed=D + d, cache=cache, nd=nd, D=D, Hq=Hq, Hkv=Hkv, d=d,
                             block=block, extra=WIDE // block)
    assert st == 0
    check(o, ls, refs, nd, rows=np.r_[0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 200, D - 2, D - 1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("row_stride", [64, 65])
def test_draft_positions_under_wide_tables(ssd, d, row_stride):  # noqa: F811
    D = 50
    rng = np.random.default_rng(d)
    pos = rng.integers(0, 400, (3, D))
    pos[0] = 150 + np.arange(D)
    pos[1, 1] = pos[1, 0]
    pos[2, 0], pos[2, 2] = -1, 64 * 64
    nd = [D, D, D - 3]
    o, ls, st, refs = attend(ssd, seed=d, cache=[153, 200, 60], nd=nd, D=D, Hq=4, Hkv=2, d=d, block=64,
                             draft_pos=pos, grid=(64, 64, 3, row_stride), extra=WIDE // 64)
    assert st == 6  # the two drafts outside the grid
    check(o, ls, refs, nd)
    assert (o[2, 0] == 0).all() and torch.isinf(ls[2, :, 2]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("extra", [0, WIDE // 32])
def test_many_drafts_with_positions(ssd, d, extra):  # noqa: F811
    """More than 512 drafts, in raster order and in none."""
    D, rng = 530, np.random.default_rng(d)
    pos = np.stack([150 + np.arange(D), rng.permutation(4000)[:D]])
    o, ls, st, refs = attend(ssd, seed=d, cache=[153, 90], nd=[D, D - 9], D=D, Hq=4, Hkv=2, d=d, block=32,
                             draft_pos=pos, extra=extra)
    assert st == 0
    check(o, ls, refs, [D, D - 9], rows=np.r_[0, 1, 2, 100, 255, 256, 400, 511, 512, D - 10, D - 1])


@pytest.mark.parametrize("d", [64, 128])
def test_masks_scales_and_blocks_under_wide_tables(ssd, d):  # noqa: F811
    D, kw = 40, dict(Hq=4, Hkv=2, d=d, block=16, extra=WIDE // 16)
    cache, nd = [200, 200, 200, 200, 50], [D] * 5
    start = [0, 17, 200 + D // 2, 200 + D, 2 ** 31 - 1]
    o, ls, st, refs = attend(ssd, seed=d, cache=cache, nd=nd, D=D, key_start=start, **kw)
    assert st == 0
    check(o, ls, refs, nd)
    assert (o[3] == 0).all() and (o[4] == 0).all() and torch.isinf(ls[3]).all()
    for other in (dict(spread=4.0), dict(peaky=8.0), dict(q_std=1e-20), dict(spread=0.0, scale=0.3)):
        o, ls, st, refs = attend(ssd, seed=d, cache=[500, 130], nd=[D, D], D=D, **kw, **other)
        assert st == 0
        check(o, ls, refs, [D, D])

    def edit(table):
        table[0, 1], table[1, 0] = -1, 10 ** 6
    o, ls, st, refs = attend(ssd, seed=2, cache=[100, 30], nd=[D, D], D=D, table_edit=edit, **kw)
    assert st == 6
    refs[0][2][:, 16:32] = False
    refs[1][2][:, 0:16] = False
    check(o, ls, refs, [D, D])


# B sequences for 3 x 152 / Hkv CTAs a head: equal lengths that do not come out even (14 and 57
# CTAs), ragged ones, some empty, one far longer than the rest, and more sequences than CTAs
@pytest.mark.parametrize("Hkv,G,d,block,lens", [
    (32, 1, 64, 64, [2500] * 8),
    (32, 4, 64, 128, [2500] * 9 + [1, 0, 700]),
    (8, 2, 128, 32, [1900] * 40),
    (8, 1, 64, 16, [0, 3000, 64, 63, 65] * 6 + [20000]),
    (8, 12, 64, 64, list(range(1, 3000, 97))),
    (24, 1, 64, 64, [700, 5000] * 12),
    (16, 8, 128, 64, [129] * 40),
])
def test_sequences_cut_for_the_whole_gpu(ssd, Hkv, G, d, block, lens):  # noqa: F811
    B, Hq, D = len(lens), Hkv * G, 1
    gen = torch.Generator("cuda").manual_seed(len(lens) * Hkv + d)
    nd = torch.tensor([0 if n == 0 else 1 for n in lens])
    need = [-(-(n + 1) // block) if n else 0 for n in lens]
    pool, M = sum(need) + 1, max(need) + 3
    ids = torch.randperm(pool, generator=gen, device="cuda")
    table = torch.full((B, M), -1, device="cuda", dtype=torch.int64)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]

    def values():
        x = torch.randn((pool, Hkv, block, d), generator=gen, device="cuda") * 100
        return x.clamp(-448, 448).to(torch.float8_e4m3fn)

    k, v = values(), values()
    ks, vs = (0.01 * torch.exp(0.5 * torch.randn((pool, Hkv), generator=gen, device="cuda"))
              for _ in range(2))
    q = torch.randn((B, D, Hq, d), generator=gen, device="cuda").to(torch.bfloat16)
    o = torch.full((B, D, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ls = torch.full((B, Hq, D), 7.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    wb = ssd.ssd_cache_attention_workspace(B, Hq, Hkv, d, D, M * block)
    ws = torch.full((max(wb, 16),), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        ssd.ssd_cache_attention(ssd.grid(64, 64, 3), ssd.cache(k, v, ks, vs), B, Hq, i32(lens), i32(nd),
                                None, None, D, table.to(torch.int32), M, q, 0.0, o, ls, ws, wb, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
    for b in range(B):
        if lens[b] == 0:
            assert (o[b] == 7).all() and (ls[b] == 7).all()
            continue
        t, L = table[b, :need[b]], lens[b] + 1

        def kept(x, s):  # [Hkv, L, d]
            y = x[t].double() * s[t].double()[:, :, None, None]
            return y.transpose(0, 1).reshape(Hkv, -1, d)[:, :L]

        kk, vv = kept(k, ks), kept(v, vs)
        sv = vs[t].double().repeat_interleave(block, 0)[:L].t()       # [Hkv, L]
        qq = q[b, 0].double().view(Hkv, G, d)
        x = torch.einsum("hgd,hld->hgl", qq, kk) * d ** -0.5
        m = x.amax(-1, keepdim=True)
        e = torch.exp(x - m)
        z = e.sum(-1, keepdim=True)
        ref = torch.einsum("hgl,hld->hgd", e / z, vv)
        A = torch.einsum("hgl,hld->hgd", e / z, vv.abs())
        F = torch.einsum("hl,hld->hd", sv.amax(-1, keepdim=True) / sv, vv.abs())[:, None] / z
        mag = qq.abs().amax(-1) * kk.abs().sum(-1).amax(-1, keepdim=True) * d ** -0.5
        off = 2.0 ** -16 * mag
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * off[..., None]) * A + 2.0 ** -16 * F + 1e-30
        err = (o[b, 0].double().view(Hkv, G, d) - ref).abs()
        assert (err <= tol).all(), (b, float((err / tol).max()))
        lse = (m + torch.log(z))[..., 0]
        assert ((ls[b, :, 0].double().view(Hkv, G) - lse).abs() <= off + 2.0 ** -17 * (1 + lse.abs())).all()
