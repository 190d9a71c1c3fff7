"""ssd_cache_attention_shared against float64 attention over each sequence's keys; tolerances are
those of the attention without groups (tests/test_gpu_cache_attention.py), whose parts it joins in
float32.  Small batches share here, too (ssd_set_cache_sharing), but for the tests of the rule; `shares`
asks the workspace's size which path it is."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache_attention import check, i32

pytestmark = pytest.mark.gpu


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


class Batch:
    """Groups of sequences over one pool: start [groups + 1], shared blocks of a group, own tokens
    (cached behind the shared ones) and drafts of a sequence.  Dead entries and unused scales NaN."""

    def __init__(self, *, seed, start, shared, own, nd, D, Hq, Hkv, d, block, wide=None, spread=0.5,
                 edit=None, grid=(64, 64, 3, 64), draft_pos=None, key_start=None, max_shared=None,
                 offset=0):
        rng = np.random.default_rng(seed)
        self.__dict__.update(start=start, shared=shared, nd=nd, D=D, Hq=Hq, Hkv=Hkv, d=d, block=block,
                             grid=grid, draft_pos=draft_pos, key_start=key_start, offset=offset)
        self.B, self.groups = len(own), len(shared)
        names, n, self.cache = [], 0, []
        for g in range(self.groups):
            first = list(range(n, n + shared[g]))
            n += shared[g]
            for b in range(start[g], start[g + 1]):
                self.cache.append(shared[g] * block + own[b])
                more = max(0, -(-(self.cache[b] + max(nd[b], 0)) // block) - shared[g])
                names.append(first + list(range(n, n + more)))
                n += more
        pool = n + 2
        ids = rng.permutation(pool)
        self.M = max(max(len(x) for x in names), 1) + (2000 if wide is None else wide)
        self.max_shared = max(max(shared), 0) if max_shared is None else max_shared
        self.table = np.full((self.B, self.M), -1)
        for b, x in enumerate(names):
            self.table[b, :len(x)] = ids[x]
        self.codes = {x: np.full((pool, Hkv, block, d), 0x7f, np.uint8) for x in "kv"}
        self.scales = {x: np.full((pool, Hkv), np.nan, np.float32) for x in "kv"}
        live = np.zeros(pool, int)
        for b in range(self.B):
            L = self.cache[b] + max(nd[b], 0)
            for i in range(len(names[b])):
                live[self.table[b, i]] = min(block, L - i * block)
        for x in "kv":
            for blk in np.nonzero(live)[0]:
                self.scales[x][blk] = np.exp(rng.normal(0, spread, Hkv)) / 100
                c = rng.standard_normal((Hkv, live[blk], d)) * 100
                c *= rng.choice([1.0, 1.0, 1.0, 2e-4, 0.0], size=(Hkv, live[blk], 1))
                t = torch.from_numpy(c.astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn)
                self.codes[x][blk, :, :live[blk]] = t.view(torch.uint8).numpy()
        self.q = torch.from_numpy(rng.standard_normal((self.B, D, Hq, d)).astype(np.float32)).to(torch.bfloat16)
        if edit is not None:
            edit(self)

    def run(self, ssd, stream=None, lse=True, twice=True):
        B, D, Hq, Hkv, d = self.B, self.D, self.Hq, self.Hkv, self.d
        off = self.offset  # blocks of the pool before the first that is used
        dev = {x: torch.from_numpy(self.codes[x]).cuda() for x in "kv"}
        dsc = {x: torch.from_numpy(self.scales[x]).cuda() for x in "kv"}
        if off:
            dev = {x: torch.cat([t.new_full((off,) + t.shape[1:], 0x7f), t]) for x, t in dev.items()}
            dsc = {x: torch.cat([t.new_full((off,) + t.shape[1:], float("nan")), t]) for x, t in dsc.items()}
        H, W, prefix, rs = self.grid
        o = torch.full((B, D, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        ls = torch.full((B, Hq, D), 7.0, device="cuda") if lse else None
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        wb = ssd.ssd_cache_attention_shared_workspace(B, self.groups, Hq, Hkv, d, D, self.M * self.block,
                                                      self.max_shared * self.block)
        ws = torch.full((max(wb, 16),), 0xff, dtype=torch.uint8, device="cuda")
        self.shares = wb != ssd.ssd_cache_attention_workspace(B, Hq, Hkv, d, D, self.M * self.block)
        opt = lambda x: None if x is None else i32(x)  # noqa: E731
        self.args = (ssd.grid(H, W, prefix, rs), ssd.cache(dev["k"], dev["v"], dsc["k"], dsc["v"]), B,
                     self.groups, i32(self.start), i32(self.shared), self.max_shared, Hq, i32(self.cache),
                     i32(self.nd), opt(self.draft_pos), opt(self.key_start), D,
                     i32(np.where(self.table >= 0, self.table + off, -1)), self.M,
                     self.q.cuda(), 0.0, o, ls, ws, wb, st)
        self.held = dev, dsc
        torch.cuda.synchronize()
        ssd.ssd_cache_attention_shared(*self.args, stream=stream)
        torch.cuda.synchronize()
        if twice:
            first = o.clone()
            ssd.ssd_cache_attention_shared(*self.args, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(first.view(torch.int16), o.view(torch.int16)), "a repeated call differs"
        return o, ls, int(st.item())

    def refs(self):
        H, W, prefix, rs = self.grid
        out = []
        for b in range(self.B):
            n, cl = max(self.nd[b], 0), self.cache[b]
            L = cl + n
            ids = self.table[b, np.arange(L) // self.block]
            at = np.arange(L) % self.block
            per = {}
            for x in "kv":
                t = torch.from_numpy(self.codes[x][ids, :, at]).view(torch.float8_e4m3fn).double().numpy()
                per[x] = t * self.scales[x][ids].astype(np.float64)[:, :, None]
            per["vs"] = self.scales["v"][ids].astype(np.float64)
            kp, qp = np.arange(L), cl + np.arange(n)
            if self.draft_pos is not None:
                i = np.asarray(self.draft_pos[b])[:n]
                inside = (i >= 0) & (i < H * W)
                qp = np.where(inside, prefix + i // W * rs + i % W, -1)
                kp = np.concatenate([kp[:cl], np.where(inside, qp, 1 << 40)])
            s0 = 0 if self.key_start is None else int(self.key_start[b])
            see = (kp[None] <= qp[:, None]) & (np.arange(L)[None] >= s0)
            out.append((self.q[b, :n].double().numpy(), per, see, self.d ** -0.5))
        return out

    def check(self, ssd, status=0, shares=True, **kw):
        o, ls, st = self.run(ssd)
        assert st == status and self.shares == shares
        check(o, ls, self.refs(), self.nd, **kw)
        return o, ls


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (8, 2, 128), (3, 1, 128)])
def test_one_token_each(ssd, block, Hq, Hkv, d):
    """Groups of many, of one and of none; one that shares nothing; own keys of every length."""
    own = [0, 1, 15, 16, 63, 64, 65, 127, 300, 0, 700, 5]
    Batch(seed=block + d, start=[0, 9, 9, 10, 12], shared=[7, 2, 5, 0], own=own, nd=[1] * 12, D=1, Hq=Hq,
          Hkv=Hkv, d=d, block=block).check(ssd)


@pytest.mark.parametrize("D", [2, 5, 16, 17, 48, 65, 130])
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 128), (8, 2, 128), (6, 2, 64)])
def test_drafts_of_every_count(ssd, D, Hq, Hkv, d):
    nd = [D, max(1, D - 1), D // 2, 0, D, 1, D]
    Batch(seed=D, start=[0, 5, 7], shared=[5, 11], own=[70, 0, 133, 9, 31, 250, 3], nd=nd, D=D, Hq=Hq, Hkv=Hkv,
          d=d, block=32).check(ssd)


@pytest.mark.parametrize("G", [1, 4, 16, 40, 129])
def test_shared_heads(ssd, G):
    Batch(seed=G, start=[0, 5], shared=[9], own=[100, 37, 0, 5, 64], nd=[3, 2, 1, 3, 0], D=3, Hq=2 * G, Hkv=2,
          d=128, block=16).check(ssd)


@pytest.mark.parametrize("row_stride", [64, 65])
@pytest.mark.parametrize("D,Hq,Hkv", [(3, 4, 2), (40, 4, 4)])
def test_draft_positions_in_any_order(ssd, row_stride, D, Hq, Hkv):
    """Positions among the shared keys and below all of them, and two outside the grid."""
    rng = np.random.default_rng(D)
    pos = rng.integers(0, 400, (4, D))
    pos[0], pos[1, 0], pos[1, 1] = 150 + np.arange(D), 0, 130
    b = Batch(seed=D, start=[0, 4], shared=[8], own=[25, 72, 0, 10], nd=[D, D, D, D - 1], D=D, Hq=Hq, Hkv=Hkv,
              d=128, block=16, draft_pos=pos, grid=(64, 64, 3, row_stride))
    b.check(ssd)
    pos[2, 0], pos[2, 2] = -1, 64 * 64
    o, ls = b.check(ssd, status=6)
    assert (o[2, 0] == 0).all() and torch.isinf(ls[2, :, 2]).all()


@pytest.mark.parametrize("D", [1, 5, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_padding_on_the_left_and_rows_that_see_nothing(ssd, D, d):
    own, nd = [50, 50, 50, 50, 0, 20], [D] * 6
    start = [0, 17, 128, 178 + D, 2 ** 31 - 1, 140]   # within the shared keys, at their end, behind all
    o, ls = Batch(seed=D, start=[0, 6], shared=[8], own=own, nd=nd, D=D, Hq=4, Hkv=2, d=d, block=16,
                  key_start=start).check(ssd)
    assert (o[3] == 0).all() and (o[4] == 0).all() and torch.isinf(ls[3]).all()


@pytest.mark.parametrize("D,Hq,Hkv,d", [(1, 8, 2, 128), (1, 2, 2, 64), (40, 2, 2, 128)])
def test_long_prompts(ssd, D, Hq, Hkv, d):
    """Shared keys of many parts beside short ones."""
    Batch(seed=D + d, start=[0, 4, 9], shared=[320, 3], own=[200, 37, 4000, 0, 0, 900, 64, 63, 1], nd=[D] * 9,
          D=D, Hq=Hq, Hkv=Hkv, d=d, block=64).check(ssd, rows=[0, 1, 17, D - 1])


@pytest.mark.parametrize("B,groups,D", [(64, 1, 1), (70, 5, 1), (300, 70, 1), (40, 33, 20)])
def test_many_sequences_and_groups(ssd, B, groups, D):
    rng = np.random.default_rng(B)
    start = [0] + sorted(rng.choice(np.arange(1, B), groups - 1, replace=False).tolist()) + [B]
    Batch(seed=B, start=start, shared=rng.integers(0, 9, groups).tolist(), own=rng.integers(0, 200, B).tolist(),
          nd=rng.integers(0, D + 1, B).tolist(), D=D, Hq=4, Hkv=1, d=64, block=16,
          wide=20000).check(ssd, rows=[0, D - 1])


@pytest.mark.parametrize("D,Hq,Hkv,d", [(1, 4, 2, 128), (1, 2, 2, 64), (2, 8, 4, 64), (3, 6, 2, 128)])
@pytest.mark.parametrize("how", ["", "key_start", "draft_pos"])
def test_few_rows_of_most_groups_and_many_of_one(ssd, D, Hq, Hkv, d, how):
    """Shared keys on the kernel for few rows: a group of 23 sequences beside ten of one or none, some
    sequences without drafts, padding, drafts anywhere on the grid."""
    rng = np.random.default_rng(D + d)
    start = [0, 1, 24, 24, 25, 26, 27, 28, 29, 30, 31, 32]
    shared = [9, 40, 5, 0, 17, 1, 3, 8, 2, 12, 64]
    B = start[-1]
    nd = [int(x) for x in rng.integers(0, D + 1, B)]
    nd[1], nd[0] = 0, D  # (the first of the long group has nothing to do)
    kw = {}
    if how == "key_start":
        kw["key_start"] = [int(x) for x in rng.integers(0, 40, B)]
    if how == "draft_pos":  # over a grid that reaches from the prompts to behind all tokens
        kw["grid"] = (64, 64, 0, 64)
        kw["draft_pos"] = rng.integers(600, 4096, (B, D))
    Batch(seed=D, start=start, shared=shared, own=[int(x) for x in rng.integers(0, 90, B)], nd=nd, D=D, Hq=Hq,
          Hkv=Hkv, d=d, block=16, **kw).check(ssd)


def test_offsets_beyond_32_bits(ssd):
    """Blocks behind the first 3 GB of a pool."""
    for D in (1, 40):
        Batch(seed=D, start=[0, 4], shared=[5], own=[100, 3, 64, 0], nd=[D] * 4, D=D, Hq=4, Hkv=2, d=128, block=64,
              offset=200000).check(ssd)


@pytest.mark.parametrize("B", [255, 256, 257, 300])
def test_groups_of_many(ssd, B):
    """Up to 256 sequences have only their drafts stacked."""
    rng = np.random.default_rng(B)
    Batch(seed=B, start=[0, B], shared=[9], own=rng.integers(0, 60, B).tolist(), nd=rng.integers(0, 3, B).tolist(),
          D=2, Hq=4, Hkv=2, d=64, block=16).check(ssd, rows=[0, 1], heads=[1, 2])


@pytest.mark.parametrize("wide", [400, 4000])
@pytest.mark.parametrize("B,Hq,Hkv,D", [(64, 16, 8, 1), (60, 8, 8, 2), (300, 4, 2, 1), (40, 24, 12, 3)])
def test_more_sequences_than_places(ssd, B, Hq, Hkv, D, wide):
    """A CTA for every sequence and head, the longest first (up to 256 sequences)."""
    rng = np.random.default_rng(B)
    start = [0, 1, B // 3, B]
    Batch(seed=B, start=start, shared=[2, 0, 11], own=rng.integers(0, 500, B).tolist(),
          nd=rng.integers(0, D + 1, B).tolist(), D=D, Hq=Hq, Hkv=Hkv, d=64, block=16,
          wide=wide).check(ssd, rows=[0, D - 1])


def test_where_sharing_pays(ssd):
    """The rule by sizes, the same results on both sides of it."""
    ssd.ssd_set_cache_sharing(0)
    small = dict(seed=3, start=[0, 2, 4], shared=[12, 12], own=[10, 200, 77, 0], nd=[1] * 4, D=1, Hq=8, Hkv=8, d=64,
                 block=16, wide=0)
    Batch(**small).check(ssd, shares=False)
    Batch(**dict(small, shared=[0, 0])).check(ssd, shares=False)
    large = dict(seed=3, start=[0, 48], shared=[40], own=list(range(48)), nd=[1] * 48, D=1, Hq=8, Hkv=8, d=64,
                 block=128, wide=0)
    Batch(**large).check(ssd, rows=[0], heads=[0, 5])
    ssd.ssd_set_cache_sharing(2)
    Batch(**large).check(ssd, shares=False, rows=[0], heads=[0, 5])
    ssd.ssd_set_cache_sharing(1)
    Batch(**small).check(ssd)
    for how in (-1, 3):
        with pytest.raises(ssd.SsdError):
            ssd.ssd_set_cache_sharing(how)


def test_scales_that_differ(ssd):
    for D in (1, 48):
        Batch(seed=D, start=[0, 3], shared=[6], own=[100, 30, 64], nd=[D] * 3, D=D, Hq=4, Hkv=2, d=128, block=16,
              spread=4.0).check(ssd)


def test_a_nan_key_reaches_the_rows_that_see_it(ssd):
    """One of the shared keys of one head: the rows of its head whose keys begin before it."""
    def edit(b):
        b.codes["k"][b.table[0, 2], 1, 3, 5] = 0x7f

    for D in (1, 40):
        b = Batch(seed=D, start=[0, 3, 5], shared=[6, 6], own=[10, 20, 30, 40, 50], nd=[D] * 5, D=D, Hq=4, Hkv=2,
                  d=128, block=16, edit=edit, key_start=[0, 0, 36, 0, 0])
        o, ls, st = b.run(ssd)
        assert st == 0 and b.shares
        nan = torch.isnan(o).all(-1)
        want = torch.zeros_like(nan)
        want[:2, :, 2:] = True
        assert torch.equal(nan, want) and torch.equal(torch.isnan(o).any(-1), want)
        assert torch.equal(torch.isnan(ls), want.transpose(1, 2))


def test_padding_of_a_shared_prompt_may_be_anything(ssd):
    """Before the first token that any sequence of the group may see: NaN in keys, values and scales."""
    for D, start in ((1, [40] * 4), (1, [64, 37, 100, 51]), (40, [40] * 4), (40, [33, 64, 34, 90]), (1, [128] * 4)):
        def edit(b):
            n = min(start)
            for i in range(-(-n // b.block)):
                for x in "kv":
                    b.codes[x][b.table[0, i], :, :n - i * b.block] = 0x7f
                    if (i + 1) * b.block <= n:
                        b.scales[x][b.table[0, i]] = np.nan

        b = Batch(seed=D, start=[0, 4], shared=[8], own=[10, 20, 30, 0], nd=[D] * 4, D=D, Hq=4, Hkv=2, d=128,
                  block=16, edit=edit, key_start=start)
        o, ls, st = b.run(ssd)
        assert st == 0 and b.shares
        refs = b.refs()
        for _, per, _, _ in refs:
            for x in per:
                per[x][:min(start)] = 0.0  # (that nobody sees)
        check(o, ls, refs, b.nd)


def test_the_first_of_a_group_may_be_done(ssd):
    """Blocks are named by a sequence that has drafts, not by one whose table is gone."""
    for D in (1, 33):
        def edit(b):
            b.table[0] = -1
            b.table[2] = 10 ** 8
            b.cache[0] = b.cache[2] = 0

        b = Batch(seed=D, start=[0, 4], shared=[6], own=[10, 20, 30, 40], nd=[0, D, 0, D], D=D, Hq=4, Hkv=2,
                  d=128, block=32, edit=edit)
        o, ls, st = b.run(ssd)
        assert st == 0 and b.shares and (o[0] == 7).all() and (o[2] == 7).all()
        refs = b.refs()
        for i in (1, 3):
            check(o[i:i + 1], ls[i:i + 1], refs[i:i + 1], [D])


def test_bad_groups_lengths_and_blocks(ssd):
    base = dict(seed=1, start=[0, 3, 5], shared=[3, 4], own=[10, 20, 5, 4, 9], D=3, Hq=4, Hkv=2, d=128, block=16)
    # fewer tokens than the group shares, more drafts than D, a negative length
    def edit(b):
        b.cache[1] = 47
        b.cache[4] = -2
    b = Batch(nd=[3, 3, 9, 3, 3], edit=edit, **base)
    o, ls, st = b.run(ssd)
    assert st == 6 and b.shares and (o[1] == 7).all() and (o[2] == 7).all() and (o[4] == 7).all()
    b.nd, b.cache[1], b.cache[4] = [3, 3, 3, 3, 3], 68, 73
    refs = b.refs()
    for i in (0, 3):
        check(o[i:i + 1], ls[i:i + 1], refs[i:i + 1], [3])
    # blocks that are shared beyond max_shared, or fewer than none
    for shared in (10 ** 9, -1):
        b = Batch(nd=[3] * 5, **base)
        b.shared = [3, b.max_shared + 1 if shared > 0 else shared]
        o, ls, st = b.run(ssd)
        assert st == 6 and (o[3:] == 7).all()
        check(o[:3], ls[:3], b.refs()[:3], [3] * 3)
    # groups that do not cover the batch, or do not ascend
    for start in ([0, 3, 4], [1, 3, 5], [0, 6, 5], [0, -7, 5]):
        b = Batch(nd=[3] * 5, **base)
        b.start = start
        assert b.run(ssd, twice=False)[2] == 6 and b.shares
    # a shared block outside the pool hides its tokens
    for D in (2, 40):
        def hide(b):
            b.table[:3, 1] = 10 ** 6
        b = Batch(seed=D, start=[0, 3], shared=[3], own=[10, 20, 5], nd=[D] * 3, D=D, Hq=4, Hkv=2, d=128, block=16)
        refs = b.refs()
        hide(b)
        o, ls, st = b.run(ssd)
        assert st == 6 and b.shares
        for r in refs:
            r[2][:, 16:32] = False
        check(o, ls, refs, [D] * 3)


def test_another_stream_graphs_and_no_lse(ssd):
    """Two captured calls with workspaces of their own, replayed side by side."""
    s = torch.cuda.Stream()
    runs = []
    for D in (1, 40):
        b = Batch(seed=4 + D, start=[0, 3], shared=[9], own=[30, 0, 77], nd=[D] * 3, D=D, Hq=4, Hkv=2, d=128, block=32)
        o, _, st = b.run(ssd, stream=s, lse=False)
        assert st == 0 and b.shares
        check(o, None, b.refs(), b.nd)
        want = o.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ssd.ssd_cache_attention_shared(*b.args)
        o.fill_(7.0)
        runs.append((b, o, want, graph, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for _, _, _, graph, stream in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, o, want, _, _ in runs:
        assert torch.equal(o.view(torch.int16), want.view(torch.int16))


def test_workspace_and_refusals(ssd):
    b = Batch(seed=1, start=[0, 3], shared=[3], own=[1, 2, 3], nd=[1] * 3, D=1, Hq=4, Hkv=2, d=64, block=16)
    b.run(ssd)
    a = list(b.args)
    assert b.shares
    for i, x in ((3, 0), (6, b.M + 1), (6, -1), (20, a[20] - 1), (4, None), (5, None)):
        bad = list(a)
        bad[i] = x
        with pytest.raises(ssd.SsdError):
            ssd.ssd_cache_attention_shared(*bad)


@pytest.mark.parametrize("D,Hq,Hkv", [(1, 8, 2), (1, 4, 4), (40, 4, 2)])
def test_two_calls_at_once(ssd, D, Hq, Hkv):
    """Calls on two streams, each with a workspace of its own, give what each gives alone."""
    calls = []
    for seed, n in ((1, 6), (2, 40)):
        own = [20 + 31 * i % 400 for i in range(n)]
        b = Batch(seed=seed, start=[0, n // 3, n], shared=[30, 60], own=own, nd=[D] * n, D=D, Hq=Hq, Hkv=Hkv,
                  d=128, block=16)
        o, ls, st = b.run(ssd)
        assert st == 0 and b.shares
        calls.append((b, o.clone(), ls.clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for b, _, _, stream in calls:
            ssd.ssd_cache_attention_shared(*b.args, stream=stream)
    torch.cuda.synchronize()
    for b, o, ls, _ in calls:
        now, lse, st = b.args[17], b.args[18], b.args[21]
        assert st.item() == 0 and torch.equal(now.view(torch.int16), o.view(torch.int16)) and torch.equal(lse, ls)
