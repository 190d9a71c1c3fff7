"""ssd_cache_plan, ssd_rotary_table and ssd_cache_append against their float64
definitions (oracle/cache.py).

Tolerances: the plan is whole numbers, equal.  The rotated q is rounded once to
bf16 (2^-8 of it) from float32 values with three roundings of 2^-24 each of |x| + |y|.  A
scale is a float32 quotient of a float32 maximum: 2^-22 relative.  An entry is
a neighbour of its unrounded value: half the e4m3 step, widened by 2^-20 of the value for
the float32 roundings before it."""
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


def run_plan(ssd, g, block, M, N, cache, new, held, ring, head, tail, table, pos=True, stream=None):
    B = len(cache)
    t = i32(table).contiguous()
    i64 = lambda v: torch.tensor([v], dtype=torch.int64, device="cuda")  # noqa: E731
    nxt, nb = i64(-5), torch.full((B,), -5, dtype=torch.int32, device="cuda")
    slots = torch.full((B, N), -5, dtype=torch.int64, device="cuda")
    p = torch.full((B, N, 3), -5, dtype=torch.int32, device="cuda") if pos else None
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ssd.ssd_cache_plan(g, B, block, M, N, i32(cache), i32(new), i32(held), i32(ring), len(ring),
                       i64(head), i64(tail), nxt, t, nb, slots, p, st)
    torch.cuda.synchronize()
    return (t.cpu().numpy(), nb.cpu().numpy(), int(nxt.item()), slots.cpu().numpy(),
            p.cpu().numpy() if pos else None, int(st.item()))


def plan_case(rng, B, N, block, spare, zero=0.1):
    cache = rng.integers(0, 900, B)
    new = rng.integers(0, N + 1, B)
    new[rng.random(B) < zero] = 0
    held = -(-cache // block) + (rng.random(B) < 0.2)      # some keep a spare block
    need = -(-(cache + new) // block)
    M = int(max(need.max(), held.max(), 1)) + 1
    demand = np.maximum(need - held, 0).sum()
    free = int(demand) + spare
    R = int(held.sum()) + max(free, 1) + 2
    ids = rng.permutation(R)
    table = np.full((B, M), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    head = 3 * R + int(rng.integers(0, R))
    ring = np.full(R, -9)
    for i in range(max(free, 0)):
        ring[(head + i) % R] = ids[at + i]
    return cache, new, held, ring, head, head + max(free, 0), table, M


@pytest.mark.parametrize("B,N,block", [(1, 1, 16), (1, 1500, 16), (3, 1023, 32), (5, 1024, 64),
                                       (2, 1025, 128), (31, 7, 16), (300, 2, 64), (700, 1, 16),
                                       (257, 4, 32), (40, 300, 16)])
@pytest.mark.parametrize("row_stride", [24, 25])
def test_plan(ssd, B, N, block, row_stride):
    rng = np.random.default_rng(B * 1000 + N)
    cache, new, held, ring, head, tail, table, M = plan_case(rng, B, N, block, 4)
    g = ssd.grid(64, 24, 50, row_stride)
    got = run_plan(ssd, g, block, M, N, cache, new, held, ring, head, tail, table)
    want = oc.plan(24, row_stride, 50, block, M, N, cache, new, held, ring, head, tail, table)
    assert got[5] == 0 and want[5].all()
    for a, b in zip(got[:5], want[:5]):
        assert np.array_equal(a, b)
    # without positions and a grid; every block dealt at most once
    again = run_plan(ssd, None, block, M, N, cache, new, held, ring, head, tail, table, pos=False)
    assert np.array_equal(again[3], want[3]) and again[2] == want[2]
    used = got[0][got[0] >= 0]
    assert len(set(used.tolist())) == len(used)


@pytest.mark.parametrize("B,N,spare", [(6, 40, -3), (300, 3, -20), (3, 1200, -30)])
def test_plan_out_of_blocks(ssd, B, N, spare):
    rng = np.random.default_rng(B)
    cache, new, held, ring, head, tail, table, M = plan_case(rng, B, N, 16, spare, zero=0.4)
    got = run_plan(ssd, ssd.grid(64, 24, 50), 16, M, N, cache, new, held, ring, head, tail, table)
    want = oc.plan(24, 24, 50, 16, M, N, cache, new, held, ring, head, tail, table)
    assert not want[5].all() and got[5] == 7
    for a, b in zip(got[:5], want[:5]):
        assert np.array_equal(a, b)


def test_plan_bad_lengths(ssd):
    rng = np.random.default_rng(3)
    cache, new, held, ring, head, tail, table, M = plan_case(rng, 8, 20, 16, 5, zero=0)
    cache[1], new[2], new[3], held[4], held[5], cache[6] = -1, -2, 21, -1, M + 1, 16 * M
    new[6] = 1
    args = (cache, new, held, ring, head, tail, table)
    got = run_plan(ssd, ssd.grid(64, 24, 50), 16, M, 20, *args)
    want = oc.plan(24, 24, 50, 16, M, 20, *args)
    assert got[5] == 6 and not want[5][1:7].any() and want[5][[0, 7]].all()
    for a, b in zip(got[:5], want[:5]):
        assert np.array_equal(a, b)
    # a ring that holds less than nothing, or more than it can
    for h, t in ((10, 9), (0, len(ring) + 1), (-1, 3)):
        got = run_plan(ssd, ssd.grid(64, 24, 50), 16, M, 20, cache, new, held, ring, h, t, table)
        assert got[5] == 6 and got[2] == h and (got[3] == -1).all()


# --------------------------------------------------------------------- rotary
def test_rotary_table(ssd):
    freq = (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    t = torch.full((5000, 64, 2), 9.0, device="cuda")
    ssd.ssd_rotary_table(5000, 64, torch.from_numpy(freq).cuda(), t)
    angle = np.arange(5000)[:, None] * freq.astype(np.float64)
    want = np.stack([np.cos(angle), np.sin(angle)], -1)
    assert np.abs(t.cpu().numpy() - want).max() <= 2.0 ** -25 + 1e-12  # rounded once


# --------------------------------------------------------------------- append
class Pool:
    """A cache whose live entries are known and whose dead ones hold garbage."""

    def __init__(self, rng, B, block, Hkv, d, cache, new, n_extra=3):
        need = [-(-(int(c) + int(n)) // block) for c, n in zip(cache, new)]
        self.n = sum(need) + n_extra
        ids = rng.permutation(self.n)
        self.M = max(max(need), 1)
        self.table = np.full((B, self.M), -1)
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
        self.block, self.B = block, B
        self.codes = {x: rng.integers(0, 256, (self.n, Hkv, block, d)).astype(np.uint8) for x in "kv"}
        self.scale = {x: np.exp(rng.normal(-5, 1, (self.n, Hkv))).astype(np.float32) for x in "kv"}
        for x in "kv":  # live entries are numbers; the rest may be NaN
            c = self.codes[x]
            for b in range(B):
                for p in range(int(cache[b])):
                    row = c[self.table[b, p // block], :, p % block]
                    row[(row & 0x7f) == 0x7f] = 0x55
        self.dev = {x: torch.from_numpy(self.codes[x].copy()).cuda() for x in "kv"}
        self.dscale = {x: torch.from_numpy(self.scale[x].copy()).cuda() for x in "kv"}

    def cache(self, ssd):
        return ssd.cache(self.dev["k"], self.dev["v"], self.dscale["k"], self.dscale["v"])

    def slots(self, cache, new, N):
        s = np.full((self.B, N), -1, np.int64)
        for b in range(self.B):
            for j in range(int(new[b])):
                p = int(cache[b]) + j
                s[b, j] = int(self.table[b, p // self.block]) * self.block + p % self.block
        return s


def bf16(rng, shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)


def append(ssd, pool, cache, new, N, Hq, x, pos, freq, sec, inter, slots=None, ld=None, in_place=False):
    """x: dict q, k, v [B, N, H, d] CPU bf16.  ld: rows of one buffer, with what lies between
    them.  Returns (q_out, status)."""
    B, Hkv, d = pool.B, x["k"].shape[2], x["k"].shape[3]
    if ld is None:
        dev = {n: t.cuda().contiguous() for n, t in x.items()}
        lds = {n: t.shape[2] * d for n, t in x.items()}
    else:
        buf = torch.full((B * N, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
        dev, at = {}, 8
        for n, h in (("v", Hkv), ("q", Hq), ("k", Hkv)):
            dev[n] = buf[:, at:at + h * d]
            dev[n].copy_(x[n].reshape(B * N, h * d))
            at += h * d + 16
        lds = {n: ld for n in x}
    n_pos = int(pos.max()) + 1
    table = torch.empty((n_pos, d // 2, 2), device="cuda")
    ssd.ssd_rotary_table(n_pos, d // 2, torch.from_numpy(freq).cuda(), table)
    q_out = dev["q"] if in_place else torch.full((B, N, Hq, d), 9.0, dtype=torch.bfloat16,
                                                 device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    s = pool.slots(cache, new, N) if slots is None else slots
    ssd.ssd_cache_append(pool.cache(ssd), ssd.rotary(table, sec, inter), B, N, Hq, i32(new),
                         torch.from_numpy(s).cuda(), i32(pos), dev["q"], lds["q"], dev["k"], lds["k"],
                         dev["v"], lds["v"], q_out, st)
    torch.cuda.synchronize()
    return q_out.float().cpu().numpy().reshape(B, N, Hq, d), int(st.item())


def check_blocks(pool, before, before_scale, name, y, cache, new):
    """Entries and scales of K or V after an append of y [B, N, Hkv, d]."""
    block = pool.block
    got = oc.TABLE[pool.dev[name].cpu().numpy()]
    scale = pool.dscale[name].cpu().numpy().astype(np.float64)
    touched = np.zeros(got.shape[0], bool)
    for b in range(pool.B):
        c, n = int(cache[b]), int(new[b])
        for i in range(c // block, -(-(c + n) // block) if n else 0):
            blk = pool.table[b, i]
            touched[blk] = True
            lo, hi = max(c, i * block), min(c + n, (i + 1) * block)
            first = lo - i * block
            for g in range(got.shape[1]):
                want, s = oc.append_block(oc.TABLE[before[blk, g]], float(before_scale[blk, g]),
                                          first, y[b, lo - c:hi - c, g])
                assert abs(scale[blk, g] - s) <= 2.0 ** -22 * s, (b, i, g)
                end = first + hi - lo
                w, e = want[:end], got[blk, g, :end]
                nan = np.isnan(w)
                assert np.array_equal(nan, np.isnan(e))
                tol = 0.5 * oc.e4m3_step(w) * (1 + 2.0 ** -20) + np.abs(w) * 2.0 ** -20
                assert (np.abs(w - e) <= tol)[~nan].all(), (name, b, i, g)
                # dead entries of a touched block are left alone
                assert np.array_equal(pool.dev[name][blk, g, end:].cpu().numpy(), before[blk, g, end:])
    assert np.array_equal(pool.dev[name].cpu().numpy()[~touched], before[~touched])
    assert np.array_equal(pool.dscale[name].cpu().numpy()[~touched], before_scale[~touched])


def one_append(ssd, seed, B, N, Hq, Hkv, d, block, cache, new, sec, inter, std=(1.0, 1.0), **kw):
    rng = np.random.default_rng(seed)
    pool = Pool(rng, B, block, Hkv, d, cache, new)
    x = dict(q=bf16(rng, (B, N, Hq, d)), k=bf16(rng, (B, N, Hkv, d), std[0]),
             v=bf16(rng, (B, N, Hkv, d), std[1]))
    pos = rng.integers(0, 700, (B, N, 3))
    freq = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    q, st = append(ssd, pool, cache, new, N, Hq, x, pos, freq, sec, inter, **kw)
    assert st == 0
    f = {n: t.double().numpy() for n, t in x.items()}
    yk = np.stack([oc.rotate(f["k"][b], pos[b], freq, sec, inter) for b in range(B)])
    for b in range(B):
        n = int(new[b])
        want = oc.rotate(f["q"][b], pos[b], freq, sec, inter)
        size = np.linalg.norm(f["q"][b], axis=-1, keepdims=True)
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * size
        assert (np.abs(q[b] - want) <= tol)[:n].all(), b
        if not kw.get("in_place"):
            assert (q[b, n:] == 9.0).all()  # padding rows
    check_blocks(pool, pool.codes["k"], pool.scale["k"], "k", yk, cache, new)
    check_blocks(pool, pool.codes["v"], pool.scale["v"], "v", f["v"], cache, new)
    # the same tokens again: nothing changes
    was = [pool.dev[n].clone() for n in "kv"] + [pool.dscale[n].clone() for n in "kv"]
    if not kw.get("in_place"):
        append(ssd, pool, cache, new, N, Hq, x, pos, freq, sec, inter, **kw)
        now = [pool.dev[n] for n in "kv"] + [pool.dscale[n] for n in "kv"]
        assert all(torch.equal(a, b) for a, b in zip(was, now))


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inter", [False, True])
def test_append_blocks_and_heads(ssd, block, d, inter):
    """Starts inside, at the first and at the last token of a block, one token and
    several blocks' worth, nothing at all."""
    cache = [0, 5, block - 1, block, 3 * block + 7, 40]
    new = [2 * block + 3, 1, 1, block, block - 7, 0]
    one_append(ssd, block + d, 6, max(new), 6, 2, d, block, cache, new, (d // 4, d // 8, d // 8),
               inter)


@pytest.mark.parametrize("Hq,Hkv,N", [(1, 1, 1), (8, 8, 1), (32, 8, 3), (5, 5, 33), (12, 4, 130)])
@pytest.mark.parametrize("sec", [(32, 0, 0), (0, 20, 12), (8, 12, 12)])
def test_append_heads_and_sections(ssd, Hq, Hkv, N, sec):
    rng = np.random.default_rng(N)
    cache, new = rng.integers(0, 100, 4), rng.integers(1, N + 1, 4)
    new[0] = N
    one_append(ssd, N, 4, N, Hq, Hkv, 64, 32, cache, new, sec, False)


def test_append_scales_grow_and_stay(ssd):
    """Large values raise the scale of what the block holds, small ones leave it."""
    for std in ((300.0, 1e-4), (1e-4, 300.0), (1e-30, 1e30)):
        one_append(ssd, 5, 3, 20, 4, 2, 128, 64, [10, 63, 100], [20, 5, 20], (64, 0, 0), False, std)


def test_append_rows_of_one_buffer_and_in_place(ssd):
    ld = (6 + 2 + 2) * 64 + 8 + 3 * 16
    one_append(ssd, 6, 2, 9, 6, 2, 64, 16, [3, 14], [9, 4], (16, 8, 8), False, ld=ld)
    one_append(ssd, 7, 2, 9, 6, 2, 64, 16, [3, 14], [9, 9], (16, 8, 8), True, in_place=True)


def test_append_zeros_nan_and_infinities(ssd):
    """All-zero tokens give a positive scale; an infinity becomes the largest
    value, a NaN stays one, and neither moves the scale."""
    rng = np.random.default_rng(8)
    pool = Pool(rng, 1, 16, 2, 64, [0], [20])
    x = dict(q=bf16(rng, (1, 20, 2, 64)), k=torch.zeros((1, 20, 2, 64), dtype=torch.bfloat16),
             v=bf16(rng, (1, 20, 2, 64)))
    x["v"][0, 3, 0, 5], x["v"][0, 4, 0, 6], x["v"][0, 17, 1, 7] = float("inf"), -float("inf"), float("nan")
    pos = np.zeros((1, 20, 3), np.int64)
    freq = np.ones(32, np.float32)
    q, st = append(ssd, pool, [0], [20], 20, 2, x, pos, freq, (32, 0, 0), False)
    assert st == 0 and np.array_equal(q, x["q"].float().numpy())
    check_blocks(pool, pool.codes["v"], pool.scale["v"], "v", x["v"].double().numpy(), [0], [20])
    check_blocks(pool, pool.codes["k"], pool.scale["k"], "k", x["k"].double().numpy(), [0], [20])
    assert (pool.dscale["k"].cpu().numpy()[pool.table[0, :2]] > 0).all()


def test_append_device_errors(ssd):
    """Lengths, slots and positions out of range are recorded and skipped."""
    rng = np.random.default_rng(9)
    freq = np.ones(32, np.float32)

    def fresh():
        pool = Pool(rng, 2, 16, 2, 64, [4, 4], [6, 6])
        x = {n: bf16(rng, (2, 6, 2, 64)) for n in "qkv"}
        return pool, x, np.zeros((2, 6, 3), np.int64)

    for new in ([6, 7], [6, -1]):
        pool, x, pos = fresh()
        was = pool.dev["k"].clone()
        q, st = append(ssd, pool, [4, 4], new, 6, 2, x, pos, freq, (32, 0, 0), False,
                       slots=pool.slots([4, 4], [6, 6], 6))
        assert st == 6 and (q[1] == 9).all()
        blk = pool.table[1, 0]
        assert torch.equal(pool.dev["k"][blk], was[blk])
    for bad in (10 ** 12, None):
        pool, x, pos = fresh()
        slots = pool.slots([4, 4], [6, 6], 6)
        if bad is None:
            slots[1, 3] += 1            # not the one after its predecessor
        else:
            slots[1, :] = bad + np.arange(6) + 4
        was = pool.dev["v"].clone()
        _, st = append(ssd, pool, [4, 4], [6, 6], 6, 2, x, pos, freq, (32, 0, 0), False, slots=slots)
        assert st == 6
        blk = pool.table[1, 0]
        same = pool.dev["v"][blk][:, 7] if bad is None else pool.dev["v"][blk]
        assert torch.equal(same, was[blk][:, 7] if bad is None else was[blk])
    pool, x, pos = fresh()
    table = torch.ones((3, 32, 2), device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.zeros((2, 6, 2, 64), dtype=torch.bfloat16, device="cuda")
    pos[1, 2] = (0, 3, 0)
    d = {n: t.cuda() for n, t in x.items()}
    ssd.ssd_cache_append(pool.cache(ssd), ssd.rotary(table, (16, 8, 8)), 2, 6, 2, i32([6, 6]),
                         torch.from_numpy(pool.slots([4, 4], [6, 6], 6)).cuda(), i32(pos), d["q"], 128,
                         d["k"], 128, d["v"], 128, out, st)
    torch.cuda.synchronize()
    assert st.item() == 6
    # a sequence that the plan could not serve: nothing is written, no error
    pool, x, pos = fresh()
    slots = pool.slots([4, 4], [6, 6], 6)
    slots[0] = -1
    was = pool.dev["k"].clone()
    q, s = append(ssd, pool, [4, 4], [6, 6], 6, 2, x, pos, freq, (32, 0, 0), False, slots=slots)
    assert s == 0 and (q[0] == 9).all()
    assert torch.equal(pool.dev["k"][pool.table[0, 0]], was[pool.table[0, 0]])
