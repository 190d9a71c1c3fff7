"""ssd_cache_attention against float64 attention over the cache's values.

Tolerances, per entry, with A, F and mag of oracle/cache.py: the output is rounded to
bf16 (8 significant bits: 2^-8 of it).  Every probability times its scale is rounded to at
least 8 significant bits, too (2^-8 of A), and to a step of 2^-16 of the row's largest (times the
largest scale) where it is small (2^-16 of F).  A score is a float32 sum over exact products of
a query kept to 2^-18 of its largest entry: its error is below 2^-16 of mag and moves its
probability by as much.  Rounding is independent from key to key, so where scores are exact to 2^-12 the
2-norm of a call's error is held to 4e-3 of the result's.  The log-sum-exp carries a score's
error and 2^-17 of itself and of one."""
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


def attend(ssd, *, seed, cache, nd, D, Hq, Hkv, d, block, draft_pos=None, key_start=None, scale=0.0,
           grid=(64, 64, 3, 64), spread=0.5, q_std=1.0, peaky=1.0, extra=0, table_edit=None,
           stream=None, lse=True, bad_values=None):
    """One call over a pool in random order whose dead entries and unused scales
    are NaN; returns (o, lse, status, reference per sequence)."""
    rng = np.random.default_rng(seed)
    B = len(cache)
    need = [-(-(int(c) + int(n)) // block) if n >= 0 and c >= 0 else 0 for c, n in zip(cache, nd)]
    pool = sum(need) + 2
    ids = rng.permutation(pool)
    M = max(max(need), 1) + extra
    table = np.full((B, M), -1)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    codes = {x: np.full((pool, Hkv, block, d), 0x7f, np.uint8) for x in "kv"}
    scales = {x: np.full((pool, Hkv), np.nan, np.float32) for x in "kv"}
    q = torch.from_numpy((rng.standard_normal((B, D, Hq, d)) * q_std).astype(np.float32))
    q = q.to(torch.bfloat16)
    vals = []
    for b in range(B):
        L = max(0, int(cache[b]) + max(0, int(nd[b])))
        per = {}
        per["vs"] = np.ones((L, Hkv))
        for x in "kv":
            per[x] = np.zeros((L, Hkv, d))
            for i in range(need[b]):
                blk = table[b, i]
                n = min(block, L - i * block)
                scales[x][blk] = np.exp(rng.normal(0, spread, Hkv)) / 100 * (peaky if x == "k" else 1)
                # values that fill the type's range, some of them zero or subnormal
                c = rng.standard_normal((Hkv, n, d)) * 100
                c *= rng.choice([1.0, 1.0, 1.0, 2e-4, 0.0], size=(Hkv, n, 1))
                t = torch.from_numpy(c.astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn)
                codes[x][blk, :, :n] = t.view(torch.uint8).numpy()
                val = t.double().numpy() * scales[x][blk].astype(np.float64)[:, None, None]
                per[x][i * block:i * block + n] = val.transpose(1, 0, 2)
                if x == "v":
                    per["vs"][i * block:i * block + n] = scales[x][blk]
        vals.append(per)
    if bad_values is not None:
        bad_values(codes, table)
    if table_edit is not None:
        table_edit(table)
    dev = {x: torch.from_numpy(codes[x]).cuda() for x in "kv"}
    dsc = {x: torch.from_numpy(scales[x]).cuda() for x in "kv"}
    c = ssd.cache(dev["k"], dev["v"], dsc["k"], dsc["v"])
    H, W, prefix, rs = grid
    g = ssd.grid(H, W, prefix, rs)
    o = torch.full((B, D, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ls = torch.full((B, Hq, D), 7.0, device="cuda") if lse else None
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    wb = ssd.ssd_cache_attention_workspace(B, Hq, Hkv, d, D, M * block)
    ws = torch.full((max(wb, 16),), 0xff, dtype=torch.uint8, device="cuda")
    dp = None if draft_pos is None else i32(draft_pos)
    ks = None if key_start is None else i32(key_start)
    args = (g, c, B, Hq, i32(cache), i32(nd), dp, ks, D, i32(table), M, q.cuda(), scale, o, ls, ws,
            wb, st)
    torch.cuda.synchronize()
    ssd.ssd_cache_attention(*args, stream=stream)
    torch.cuda.synchronize()
    first = o.clone()
    ssd.ssd_cache_attention(*args, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), o.view(torch.int16)), "a repeated call differs"
    sc = scale if scale else d ** -0.5
    refs = []
    for b in range(B):
        n, cl = int(nd[b]), int(cache[b])
        L = cl + n
        kp = np.arange(max(L, 0))
        qp = cl + np.arange(max(n, 0))
        if draft_pos is not None:
            i = np.asarray(draft_pos[b])[:max(n, 0)]
            inside = (i >= 0) & (i < H * W)
            flat = np.where(inside, prefix + i // W * rs + i % W, -1)
            qp = flat
            kp = np.concatenate([kp[:cl], np.where(inside, flat, 1 << 40)])
        s0 = 0 if key_start is None else int(key_start[b])
        see = (kp[None] <= qp[:, None]) & (np.arange(max(L, 0))[None] >= s0)
        refs.append((q[b, :max(n, 0)].double().numpy(), vals[b], see, sc))
    return o, ls, int(st.item()), refs


def check(o, ls, refs, nd, rows=None, heads=None):
    """All rows, or a sample of them, and the 2-norm over what was compared."""
    og = o.float().cpu().numpy().astype(np.float64)
    lg = None if ls is None else ls.cpu().numpy().astype(np.float64)
    num = den = worst = 0.0
    for b, (q, v, see, sc) in enumerate(refs):
        n = int(nd[b])
        js = np.arange(n) if rows is None else np.unique(np.clip(rows, 0, n - 1))
        if n == 0:
            js = np.arange(0)
        Hq = q.shape[1]
        hs = np.arange(Hq) if heads is None else np.asarray(heads)
        G = Hq // v["k"].shape[1]
        for h in hs:
            g = h // G
            ref, lse, A, F, mag = oc.attention(q[js][:, [h]], v["k"][:, [g]], v["v"][:, [g]], see[js],
                                               sc, v["vs"][:, [g]])
            got = og[b, js, h]
            err = np.abs(got - ref[:, 0])
            off = 2.0 ** -16 * mag  # of a score
            tol = (2.0 ** -8 * np.abs(ref[:, 0]) + (2.0 ** -8 + 2 * off) * A[:, 0]
                   + 2.0 ** -16 * F[:, 0] + 1e-30)
            worst = max(worst, off.max(initial=0.0))
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
            num += (err ** 2).sum()
            den += (ref ** 2).sum()
            if lg is not None:
                gl, e = lg[b, h, js], np.isinf(lse[:, 0])
                assert (gl[e] == -np.inf).all()
                t = off[:, 0] + 2.0 ** -17 * (1 + np.abs(lse[:, 0]))
                assert (np.abs(gl[~e] - lse[~e, 0]) <= t[~e]).all(), (b, h)
        assert (og[b, n:] == 7.0).all()  # padding rows untouched
    if worst <= 2.0 ** -12:
        assert num <= (4e-3) ** 2 * max(den, 1e-30)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (8, 2, 128), (3, 1, 128)])
def test_one_token_each(ssd, block, Hq, Hkv, d):
    cache = [0, 1, 15, 16, 63, 64, 65, 127, 300, 1000]
    nd = [1] * len(cache)
    o, ls, st, refs = attend(ssd, seed=block + d, cache=cache, nd=nd, D=1, Hq=Hq, Hkv=Hkv, d=d,
                             block=block)
    assert st == 0
    check(o, ls, refs, nd)


@pytest.mark.parametrize("D", [2, 5, 16, 17, 33, 48, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 128), (8, 2, 128), (6, 2, 64)])
def test_drafts_of_every_count(ssd, D, Hq, Hkv, d):
    cache = [70, 0, 333, 9]
    nd = [D, max(1, D - 1), D // 2, 0]
    o, ls, st, refs = attend(ssd, seed=D, cache=cache, nd=nd, D=D, Hq=Hq, Hkv=Hkv, d=d, block=32)
    assert st == 0
    check(o, ls, refs, nd)


@pytest.mark.parametrize("G", [1, 4, 16, 40, 129])
def test_shared_heads(ssd, G):
    o, ls, st, refs = attend(ssd, seed=G, cache=[100, 37], nd=[3, 2], D=3, Hq=2 * G, Hkv=2, d=128,
                             block=16)
    assert st == 0
    check(o, ls, refs, [3, 2])


@pytest.mark.parametrize("row_stride", [64, 65])
@pytest.mark.parametrize("D,Hq,Hkv", [(7, 4, 2), (48, 4, 4), (100, 4, 2)])
def test_draft_positions_in_any_order(ssd, row_stride, D, Hq, Hkv):
    """Positions below, above and between the cache's, repeated ones, and two that lie
    outside the grid (seen by none, seeing none)."""
    rng = np.random.default_rng(D)
    pos = rng.integers(0, 400, (3, D))
    pos[0] = 150 + np.arange(D)
    pos[1, 1] = pos[1, 0]
    o, ls, st, refs = attend(ssd, seed=D, cache=[153, 200, 60], nd=[D, D, D - 3], D=D, Hq=Hq, Hkv=Hkv,
                             d=128, block=64, draft_pos=pos, grid=(64, 64, 3, row_stride))
    assert st == 0
    check(o, ls, refs, [D, D, D - 3])
    pos[2, 0], pos[2, 2] = -1, 64 * 64
    o, ls, st, refs = attend(ssd, seed=D, cache=[153, 200, 60], nd=[D, D, D - 3], D=D, Hq=Hq, Hkv=Hkv,
                             d=128, block=64, draft_pos=pos, grid=(64, 64, 3, row_stride))
    assert st == 6
    check(o, ls, refs, [D, D, D - 3])
    assert (o[2, 0] == 0).all() and torch.isinf(ls[2, :, 2]).all()


@pytest.mark.parametrize("D", [1, 5, 40])
def test_padding_on_the_left_and_rows_that_see_nothing(ssd, D):
    cache, nd = [200, 200, 200, 200, 50], [D] * 5
    start = [0, 17, 200, 200 + D, 2 ** 31 - 1]
    if D > 1:
        start[2] = 200 + D // 2   # the first drafts see nothing
    for d, Hkv in ((128, 2), (64, 4)):
        o, ls, st, refs = attend(ssd, seed=D, cache=cache, nd=nd, D=D, Hq=4, Hkv=Hkv, d=d, block=16,
                                 key_start=start)
        assert st == 0
        check(o, ls, refs, nd)
        assert (o[3] == 0).all() and (o[4] == 0).all() and torch.isinf(ls[3]).all()


@pytest.mark.parametrize("D,Hq,Hkv,d", [(1, 8, 2, 128), (1, 2, 2, 64), (6, 4, 4, 128), (40, 2, 2, 128)])
def test_long_caches(ssd, D, Hq, Hkv, d):
    """Caches of many parts, ragged beside short ones, tables longer than needed."""
    cache, nd = [20000, 37, 8191, 4096], [D] * 4
    o, ls, st, refs = attend(ssd, seed=D + d, cache=cache, nd=nd, D=D, Hq=Hq, Hkv=Hkv, d=d, block=64,
                             extra=500)
    assert st == 0
    check(o, ls, refs, nd, rows=[0, 1, 17, D - 1])


@pytest.mark.parametrize("D", [1, 48])
def test_scales_that_differ_and_peaked_scores(ssd, D):
    """Block scales over many orders of magnitude, scores up to a few hundred, large
    and tiny queries."""
    for kw in (dict(spread=4.0), dict(peaky=8.0), dict(q_std=1e-20, peaky=1.0), dict(q_std=1e4, peaky=1e-4),
               dict(spread=0.0, scale=0.3)):
        o, ls, st, refs = attend(ssd, seed=D, cache=[500, 130], nd=[D, D], D=D, Hq=4, Hkv=2, d=128,
                                 block=16, **kw)
        assert st == 0
        check(o, ls, refs, [D, D])


@pytest.mark.parametrize("D", [1, 48])
def test_blocks_of_zeros(ssd, D):
    """Blocks whose values are zero, at the smallest scale an append gives."""
    def zero(codes, table):
        for x in "kv":
            codes[x][table[0, ::2], :, :, :] = 0

    rngs = dict(seed=3, cache=[256], nd=[D], D=D, Hq=2, Hkv=2, d=128, block=64)
    o, _, st, refs = attend(ssd, bad_values=zero, **rngs)
    for x in "kv":
        for i in range(0, -(-(256 + D) // 64), 2):
            refs[0][1][x][i * 64:(i + 1) * 64] = 0
    assert st == 0
    check(o, None, refs, [D])


def test_bad_lengths_and_blocks(ssd):
    """A sequence with bad lengths is left alone; a block id outside the pool hides its tokens."""
    nd = [3, 9, -1, 3]
    o, ls, st, refs = attend(ssd, seed=1, cache=[20, 20, 20, -4], nd=nd, D=8, Hq=2, Hkv=2, d=64, block=16)
    assert st == 6 and (o[1:] == 7).all() and (ls[1:] == 7).all()
    check(o[:1], ls[:1], refs[:1], [3])
    for D in (2, 40):
        def edit(table):
            table[0, 1], table[1, 0] = -1, 10 ** 6
        o, ls, st, refs = attend(ssd, seed=2, cache=[100, 30], nd=[D, D], D=D, Hq=2, Hkv=2, d=128,
                                 block=16, table_edit=edit)
        assert st == 6
        refs[0][2][:, 16:32] = False
        refs[1][2][:, 0:16] = False
        check(o, ls, refs, [D, D])


def test_other_streams_and_no_lse(ssd):
    s = torch.cuda.Stream()
    for D in (1, 40):
        o, _, st, refs = attend(ssd, seed=4, cache=[300], nd=[D], D=D, Hq=4, Hkv=2, d=128, block=32,
                                stream=s, lse=False)
        assert st == 0
        check(o, None, refs, [D])


def test_workspace_query_and_refusal(ssd):
    with pytest.raises(ssd.SsdError):
        attend(ssd, seed=4, cache=[10], nd=[1], D=1, Hq=3, Hkv=2, d=128, block=32)
    with pytest.raises(ssd.SsdError):
        attend(ssd, seed=4, cache=[10], nd=[1], D=1, Hq=2, Hkv=2, d=128, block=32, scale=-1.0)
