"""ssd_sample against the float64 sampler, one row at a time.

Tolerances: a float32 weight is within WEIGHT_ERR = 1e-5 of its float64 value
(oracle/sample.py) and its integer within half a unit, so a running sum over n kept
entries is within (1e-5 + n / 2^31) Z, and u Z must lie in the drawn token's interval
widened by twice that (once for the sum, once for Z).  The kept count must lie between the
counts that a cut within that error allows."""
import numpy as np
import pytest
import torch

from oracle.sample import WEIGHT_ERR, sample_row

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


def draw(ssd, x, settings, u=None, ld=None, offset=0, arrays=False, **kw):
    """x [rows, V] (float32 or bfloat16 CUDA), laid out with rows ld apart from
    element `offset` of a buffer on."""
    rows, V = x.shape
    ld = V if ld is None else ld
    buf = torch.full((offset + rows * ld,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[offset:].view(rows, ld)
    view[:, :V] = x
    tok = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((rows,), -7.0, device="cuda")
    kept = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    if arrays:
        names = ("temperatures", "top_ks", "top_ps", "min_ps")
        dts = (torch.float32, torch.int32, torch.float32, torch.float32)
        keep = {n: torch.tensor([s[i] for s in settings], dtype=t, device="cuda")
                for i, (n, t) in enumerate(zip(names, dts))}
        p = ssd.sampling(**keep, **kw)
    else:
        p = ssd.sampling(*settings, **kw)
    ssd.ssd_sample(rows, V, view, ld, p, ssd.rng(7, 3, u), tok, prob, kept, st)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), prob.cpu().numpy(), kept.cpu().numpy(), int(st.item())


def check(x, settings, u, out):
    """settings: one tuple or one for each row, as float32 values."""
    tok, prob, kept, st = out
    assert st == 0
    xs = x.float().cpu().numpy()
    exact = 0
    for r in range(xs.shape[0]):
        T, k, p, mp = settings[r] if isinstance(settings, list) else settings
        T, p, mp = (float(np.float32(v)) for v in (T, p, mp))
        ref = sample_row(xs[r], T, k, p, mp, float(u[r]))
        assert ref["lo"] <= kept[r] <= ref["hi"], (r, kept[r], ref["lo"], ref["hi"])
        if ref["kept"] <= 1 and ref["hi"] <= 1:
            assert (tok[r], prob[r]) == (ref["tok"], np.float32(ref["prob"])), r
            exact += 1
            continue
        assert tok[r] in ref["ids"], r
        exact += tok[r] == ref["tok"]
        if ref["lo"] != ref["hi"]:
            continue
        ids, cum = ref["ids"], ref["cum"]
        at = int(np.searchsorted(ids, tok[r]))
        Z, n = cum[-1], len(ids)
        tol = 2 * (WEIGHT_ERR + n / 2.0 ** 31) * Z
        lower = cum[at - 1] if at else 0.0
        assert lower - tol <= u[r] * Z <= cum[at] + tol, (r, tok[r], ref["tok"])
        w = cum[at] - lower
        assert abs(prob[r] * Z - w) <= tol * w / Z + 1.0, r
    return exact


def uniforms(rows, seed):
    u = torch.rand((rows, 2), generator=torch.Generator().manual_seed(seed))
    u[0, 1] = 0.0
    if rows > 1:
        u[1, 1] = 1 - 2.0 ** -24
    return u


@pytest.mark.parametrize("V", [1, 2, 31, 256, 257, 1000, 4096, 16384, 32771, 65536, 100003])
@pytest.mark.parametrize("settings", [(1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.3, 2000, 0.9, 0.0),
                                      (1.0, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.05), (0.9, 300, 0.8, 0.01),
                                      (0.0, 0, 1.0, 0.0), (1.0, 1, 0.5, 0.0)])
def test_rows_of_every_size(ssd, V, settings):
    rows = 7
    g = torch.Generator().manual_seed(V + 1)
    x = 2.0 * torch.randn((rows, V), generator=g)
    u = uniforms(rows, V)
    out = draw(ssd, x.cuda(), settings, u.cuda())
    assert check(x, settings, u[:, 1].double().numpy(), out) >= rows - 1


@pytest.mark.parametrize("offset,ld", [(0, 5003), (1, 5001), (3, 5004), (0, 5120)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_types_strides_and_alignment(ssd, dtype, offset, ld):
    """bf16 logits have many ties; rows start at any element."""
    rows, V = 9, 5001
    x = (2.0 * torch.randn((rows, V), generator=torch.Generator().manual_seed(1))).to(dtype)
    u = uniforms(rows, 2)
    for settings in ((1.0, 100, 0.9, 0.0), (1.0, 0, 0.5, 0.0), (1.0, 0, 1.0, 0.0)):
        out = draw(ssd, x.cuda(), settings, u.cuda(), ld=ld, offset=offset)
        assert check(x, settings, u[:, 1].double().numpy(), out) >= rows - 1


def test_settings_of_their_own_and_padding(ssd):
    rows, V, D = 24, 3000, 6
    g = np.random.default_rng(0)
    settings = [(float(g.choice([0.0, 0.5, 1.0, 1.7])), int(g.choice([0, 1, 5, 200, 4000])),
                 float(g.choice([0.2, 0.9, 1.0])), float(g.choice([0.0, 0.01, 0.3])))
                for _ in range(rows)]
    x = 2.0 * torch.randn((rows, V), generator=torch.Generator().manual_seed(3))
    u = uniforms(rows, 4)
    out = draw(ssd, x.cuda(), settings, u.cuda(), arrays=True)
    assert check(x, settings, u[:, 1].double().numpy(), out) >= rows - 1
    nd = torch.tensor([6, 0, 3, 1], dtype=torch.int32, device="cuda")
    x[6:12] = float("nan")
    got = draw(ssd, x.cuda(), settings, u.cuda(), arrays=True, n_drafts=nd, D_max=D)
    live = np.array([j < [6, 0, 3, 1][b] for b in range(4) for j in range(D)])
    for i in range(3):
        assert np.array_equal(got[i][live], out[i][live])
    assert (got[0][~live] == -1).all() and (got[1][~live] == 0).all() and (got[2][~live] == 0).all()


def test_ties_infinities_nan_and_empty_rows(ssd):
    V = 2050
    inf, nan = float("inf"), float("nan")
    x = torch.zeros((8, V))
    x[1, 5:9] = 1.0                      # four largest, the rest equal
    x[2] = -inf
    x[3] = nan
    x[4, :] = -inf
    x[4, 77] = -3e38                     # one entry alone
    x[5, [3, 900, 2049]] = inf           # infinite logits share the mass
    x[6] = torch.randn(V, generator=torch.Generator().manual_seed(5))
    x[6, ::3] = nan
    x[7] = -0.0
    x[7, ::2] = 0.0                      # -0 and +0 are equal: index order
    u = torch.full((8, 2), 0.6)
    for settings in ((1.0, 0, 1.0, 0.0), (1.0, 7, 1.0, 0.0), (1.0, 0, 0.3, 0.0), (0.0, 0, 1.0, 0.0)):
        tok, prob, kept, st = draw(ssd, x.cuda(), settings, u.cuda())
        assert st == 0
        assert tok[2] == tok[3] == -1 and prob[2] == kept[3] == 0
        assert (tok[4], prob[4], kept[4]) == (77, 1.0, 1)
        for r in (0, 1, 6, 7):
            sub = check(x[r:r + 1], settings, np.array([np.float32(0.6)], np.float64),
                        (tok[r:r + 1], prob[r:r + 1], kept[r:r + 1], 0))
            assert sub == 1, (settings, r)
    tok, _, kept, _ = draw(ssd, x.cuda(), (1.0, 7, 1.0, 0.0), u.cuda())
    assert kept[0] == 7 and tok[0] == 4      # of 0 .. 6, u = 0.6
    assert tok[7] == 4 and kept[7] == 7
    assert kept[1] == 7 and tok[1] in (5, 6, 7)
    tok, prob, kept, _ = draw(ssd, x.cuda(), (1.0, 0, 1.0, 0.0), u.cuda())
    assert (tok[5], kept[5]) == (900, 3) and prob[5] == np.float32(1 / 3)


def test_all_equal_rows_cut_by_index(ssd):
    """Every entry at the cut: top-k and top-p keep the lowest indexes."""
    V = 70001
    x = torch.full((3, V), 1.25)
    u = torch.tensor([[0, 0.999999], [0, 0.5], [0, 0.0]])
    tok, _, kept, st = draw(ssd, x.cuda(), (1.0, 12345, 1.0, 0.0), u.cuda())
    assert st == 0 and (kept == 12345).all() and list(tok) == [12344, 6172, 0]
    tok, _, kept, _ = draw(ssd, x.cuda(), (1.0, 0, 0.25, 0.0), u.cuda())
    assert (kept == -(-V // 4)).all() and tok[0] == kept[0] - 1


def test_shares_follow_the_law(ssd):
    """One row drawn at 20000 evenly spread uniforms: every token's share is its
    probability within one uniform on each side of its interval."""
    rows, V = 20000, 64
    x = torch.randn((1, V), generator=torch.Generator().manual_seed(8)) * 1.5
    u = torch.zeros((rows, 2))
    u[:, 1] = (torch.arange(rows) + 0.5) / rows
    tok, prob, kept, st = draw(ssd, x.expand(rows, V).cuda(), (0.8, 40, 0.93, 0.0), u.cuda())
    ref = sample_row(x[0].numpy(), float(np.float32(0.8)), 40, float(np.float32(0.93)), 0.0, 0.5)
    p = np.diff(np.concatenate([[0], ref["cum"]])) / ref["cum"][-1]
    share = np.bincount(tok, minlength=V)[ref["ids"]] / rows
    assert st == 0 and (kept == ref["kept"]).all()
    assert np.abs(share - p).max() <= 1.0 / rows + 2e-5
    assert np.isin(tok, ref["ids"]).all()


def test_philox_rows_and_repeated_calls(ssd):
    """Without given uniforms a row's u_res is Philox's; a call repeats itself."""
    from synth import philox_uniforms
    rows, V = 40, 9000
    x = 2.0 * torch.randn((rows, V), generator=torch.Generator().manual_seed(9))
    s = (1.0, 700, 0.97, 0.0)
    a = draw(ssd, x.cuda(), s)
    b = draw(ssd, x.cuda(), s, torch.from_numpy(philox_uniforms(7, 3, rows)).cuda())
    c = draw(ssd, x.cuda(), s)
    for i in range(3):
        assert np.array_equal(a[i], b[i]) and np.array_equal(a[i], c[i])


def test_settings_out_of_range_on_the_device(ssd):
    x = torch.randn((5, 300)).cuda()
    bad = [(-1.0, 0, 1.0, 0.0), (1.0, -2, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 1.5),
           (1.0, 0, 1.0, 0.0)]
    tok, prob, kept, st = draw(ssd, x, bad, uniforms(5, 1).cuda(), arrays=True)
    assert st == 6 and (tok[:4] == -1).all() and (kept[:4] == 0).all() and tok[4] >= 0
