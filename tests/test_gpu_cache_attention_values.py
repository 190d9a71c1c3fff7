"""ssd_cache_attention where the values are awkward: NaN and infinities in what a row sees,
and V scales that lie far apart.  Every kernel and cut: a CTA's 8 or 16 rows and the
tensor-core kernel (from 17 rows under a table for many tokens), sequences that are whole
and sequences cut into parts.

A NaN in a key's K reaches the rows that see the key, one in its V that column of them (and may
reach it in rows of the head that see other keys only); a NaN or an infinity in a query its row.
Their log-sum-exp is NaN for K and the query.  A row that sees nothing is 0 and -inf all the same.

Tolerances of the others, per entry: bf16 of the output (2^-8 of it) and of a probability (2^-8 of
A = sum p |v|), a score exact to 2^-16 of mag = max |q| * max sum |k| * scale, and probabilities
times their V scale as float16 whose largest in the row is at least one: the step below float16's
normal range is 2^-24 of that largest, times the e4m3 entries.  The V scales of keys that a row
does not see, or hardly weighs, are in none of these.  The log-sum-exp carries a score's error and
2^-17 of itself and of one."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache_attention import i32, ssd  # noqa: F401

pytestmark = pytest.mark.gpu

BLOCK = 16
# name: drafts, query heads of a KV head, cached tokens, tokens of the table
PATHS = {
    "8 rows": (1, 4, 96, 512),
    "8 rows, cut": (1, 4, 3008, 4096),
    "8 rows, row groups": (24, 1, 96, 512),
    "16 rows": (3, 4, 96, 160000),
    "16 rows, cut": (3, 4, 3008, 160000),
    "tensor cores": (24, 2, 96, 160000),
    "tensor cores, cut": (24, 2, 3008, 160000),
}


class Call:
    """One sequence of cache + D tokens, two KV heads; its cache's dead entries and unused scales
    are NaN."""

    def __init__(self, path, d, seed=1):
        self.D, self.G, self.cache, self.room = PATHS[path]
        self.d, self.Hkv = d, 2
        self.Hq = self.Hkv * self.G
        gen = torch.Generator("cuda").manual_seed(seed)
        self.L = self.cache + self.D
        self.need = -(-self.L // BLOCK)
        pool = self.need + 2

        def new(*shape):
            return torch.randn(shape, generator=gen, device="cuda")

        def codes():
            x = (100 * new(pool, self.Hkv, BLOCK, d)).clamp(-448, 448)
            return x.to(torch.float8_e4m3fn).view(torch.uint8)

        self.ids = torch.randperm(pool, generator=gen, device="cuda")
        self.table = torch.full((1, self.room // BLOCK), -1, dtype=torch.int32, device="cuda")
        self.table[0, :self.need] = self.ids[:self.need]
        self.k, self.v = codes(), codes()
        self.ks, self.vs = torch.full((pool, self.Hkv), 0.01, device="cuda"), \
            torch.full((pool, self.Hkv), 0.01, device="cuda")
        dead = self.ids[self.need:]
        for x in (self.k, self.v):
            x[dead] = 0x7f
            if self.L % BLOCK:
                x[self.ids[self.need - 1], :, self.L % BLOCK:] = 0x7f
        self.ks[dead] = self.vs[dead] = float("nan")
        self.q = new(1, self.D, self.Hq, d).to(torch.bfloat16)
        self.draft_pos = None
        self.start = 0

    def at(self, s):
        """Block and place of token s."""
        return self.ids[s // BLOCK], s % BLOCK

    def run(self, ssd):  # noqa: F811
        D, Hq, d = self.D, self.Hq, self.d
        o = torch.full((1, D, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((1, Hq, D), 7.0, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        n = ssd.ssd_cache_attention_workspace(1, Hq, self.Hkv, d, D, self.room)
        ws = torch.full((max(n, 16),), 0xff, dtype=torch.uint8, device="cuda")
        k, v = (x.view(torch.float8_e4m3fn) for x in (self.k, self.v))
        ssd.ssd_cache_attention(
            ssd.grid(64, 64, 0), ssd.cache(k, v, self.ks, self.vs), 1, Hq, i32([self.cache]), i32([D]),
            None if self.draft_pos is None else i32([self.draft_pos]), i32([self.start]), D, self.table,
            self.room // BLOCK, self.q, 0.0, o, lse, ws, n, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        return o[0].double(), lse[0].double().t()  # [D, Hq, d], [D, Hq]

    def see(self):
        """[D, L]"""
        s, j = torch.arange(self.L, device="cuda"), torch.arange(self.D, device="cuda")
        kp, qp = s, self.cache + j
        if self.draft_pos is not None:
            qp = torch.tensor(self.draft_pos, device="cuda")
            kp = torch.cat([s[:self.cache], qp])
        return (kp[None] <= qp[:, None]) & (s >= self.start)[None]

    def check(self, o, lse, rows=None):
        """Rows [D, Hq] (bool; default all) against 64 bits."""
        rows = torch.ones((self.D, self.Hq), dtype=torch.bool, device="cuda") if rows is None else rows
        t, see = self.ids[:self.need], self.see()
        for g in range(self.Hkv):
            code = {}
            for name, x in (("k", self.k), ("v", self.v)):
                y = x[t, g].view(torch.float8_e4m3fn).double().reshape(-1, self.d)[:self.L]
                code[name] = y.nan_to_num(0.0)
            ks, vs = (x[t, g].double().repeat_interleave(BLOCK)[:self.L] for x in (self.ks, self.vs))
            k, v = code["k"] * ks[:, None], code["v"] * vs[:, None]
            hs = slice(g * self.G, (g + 1) * self.G)
            q = self.q[0, :, hs].double().nan_to_num(0.0, 0.0, 0.0)      # [D, G, d]
            scale = self.d ** -0.5
            x = torch.einsum("jhd,sd->jhs", q, k) * scale
            x = x.masked_fill(~see[:, None], -torch.inf)
            m = x.amax(-1, keepdim=True)
            p = torch.exp(x - m)
            z = p.sum(-1, keepdim=True)
            p = p / z
            ref = torch.einsum("jhs,sd->jhd", p, v)
            A = torch.einsum("jhs,sd->jhd", p, v.abs())
            C = torch.einsum("js,sd->jd", see.double(), code["v"].abs())[:, None]
            P = (p * vs).amax(-1, keepdim=True)
            ksum = torch.where(see, k.abs().sum(-1)[None], 0.0).amax(-1)[:, None]
            off = 2.0 ** -16 * (q.abs().amax(-1) * ksum * scale)
            tol = (2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * off[..., None]) * A + 2.0 ** -24 * P * C
                   + 1e-30)
            use = rows[:, hs]
            err = (o[:, hs] - ref).abs()
            assert bool((err <= tol)[use].all()), (g, float((err / tol)[use].max()))
            ref_lse = (m + torch.log(z))[..., 0]
            assert bool(((lse[:, hs] - ref_lse).abs() <= off + 2.0 ** -17 * (1 + ref_lse.abs()))[use]
                        .all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("path", PATHS)
def test_nan_in_a_key(ssd, path, d):  # noqa: F811
    """Of the first KV head, in a cached token and in the last draft."""
    for s in (5, -1):
        c = Call(path, d)
        s %= c.L
        b, i = c.at(s)
        c.k[b, 0, i, 3] = 0x7f
        o, lse = c.run(ssd)
        hit = c.see()[:, s, None] & (torch.arange(c.Hq, device="cuda") < c.G)[None]
        assert bool(hit.any())
        assert bool(torch.isnan(o)[hit].all()), "a NaN key is hidden"
        assert bool(torch.isnan(lse)[hit].all())
        c.check(o, lse, ~hit)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("path", PATHS)
def test_nan_in_a_value(ssd, path, d):  # noqa: F811
    c = Call(path, d)
    b, i = c.at(7)
    c.v[b, 0, i, 9] = 0xff
    o, lse = c.run(ssd)
    head = (torch.arange(c.Hq, device="cuda") < c.G)[None]
    assert bool(torch.isnan(o[:, :c.G, 9]).all())
    o[:, :c.G, 9] = torch.nan
    assert int(torch.isnan(o).sum()) == c.D * c.G  # no other column, no other head
    assert not bool(torch.isnan(lse).any())
    c.check(o, lse, ~head.expand(c.D, -1))
    # the first draft of a sequence whose only tokens before it are padding sees itself; with all
    # tokens padded no row sees any
    c.start = 2 ** 30
    o, lse = c.run(ssd)
    assert bool((o == 0).all()) and bool((lse == -torch.inf).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
def test_a_query_that_is_not_finite(ssd, path, d, what):  # noqa: F811
    c = Call(path, d)
    j, h = c.D // 2, c.Hq - 1
    c.q[0, j, h, d - 3] = float(what)
    o, lse = c.run(ssd)
    hit = torch.zeros((c.D, c.Hq), dtype=torch.bool, device="cuda")
    hit[j, h] = True
    assert bool(torch.isnan(o[j, h]).all()) and bool(torch.isnan(lse[j, h]))
    c.check(o, lse, ~hit)
    c.start = 2 ** 30  # (sees no key)
    o, lse = c.run(ssd)
    assert bool((o == 0).all()) and bool((lse == -torch.inf).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("log2", [20, 40, 90])
def test_large_values_that_hardly_weigh(ssd, path, d, log2):  # noqa: F811
    """The first block's V are 2^log2 times the others', and its keys' scores 100 below: the row
    is what the others give (their weights are e^100 = 2^144 times as large)."""
    c = Call(path, d)
    first = c.ids[0]
    c.vs *= 2.0 ** -30
    c.vs[first] *= 2.0 ** log2
    c.q[..., 0] = 8.0
    c.k[..., 0] = 0
    c.ks[first] = 100 * d ** 0.5 / 8 / 448
    c.k[first] = 0
    c.k[first, :, :, 0] = 0xfe  # -448
    o, lse = c.run(ssd)
    c.check(o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("step", [-5.0, 5.0, 0.0])
def test_value_scales_that_rise_and_fall(ssd, path, d, step):  # noqa: F811
    """By 2^step from block to block (up to 2^60), or zero for every other block."""
    c = Call(path, d)
    i = torch.arange(c.need, device="cuda")
    c.vs[c.ids[:c.need]] *= torch.exp2(step * i.clamp(max=12))[:, None]
    if step == 0.0:
        c.vs[c.ids[:c.need:2]] = 0.0
    o, lse = c.run(ssd)
    c.check(o, lse)
    c.vs[c.ids[:c.need]] = 0.0
    o, lse = c.run(ssd)
    assert bool((o == 0).all())
    c.check(o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("path", [p for p in PATHS if PATHS[p][0] > BLOCK])
def test_large_values_of_drafts_that_are_not_seen(ssd, path, d):  # noqa: F811
    """The first 16 drafts come behind the others in the grid and have V 2^40 times as large."""
    c = Call(path, d)
    n = c.D - BLOCK
    c.draft_pos = list(range(c.cache + n, c.cache + c.D)) + list(range(c.cache, c.cache + n))
    c.vs *= 2.0 ** -30
    c.vs[c.ids[c.cache // BLOCK]] *= 2.0 ** 40
    o, lse = c.run(ssd)
    c.check(o, lse)
