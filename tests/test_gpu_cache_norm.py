"""ssd_cache_append_norm against its float64 definition (oracle/cache.py).

Tolerances.  A head's sum of d <= 128 squares (or values) is made of at most 16 + 3 additions in
float32, so 1 / sqrt of it is off by at most (19 / 2 + 4) 2^-24 < 2^-20 relative; a mean by 2^-19 of
the mean magnitude.  y = x r gain + bias adds three roundings, the rotation three of the pair's
|a| + |b|.  In all less than e = 2^-18 (|pair| + |bias| + r |gain| mean |x|), the last for layer norms.
q is rounded to bf16 (half a step: 2^-8 of it).  A scale
carries e of its largest entry; an entry of K half the e4m3 step beside e over the scale."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.test_gpu_cache import Pool, bf16, check_blocks, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


def make_norm(rng, Hq, Hkv, d, per_head, bias, gain=True):
    out = {}
    for n, h in (("q", Hq), ("k", Hkv)):
        shape = (h, d) if per_head else (d,)
        out[n + "_gain"] = (1 + 0.3 * rng.standard_normal(shape)).astype(np.float32) if gain else None
        out[n + "_bias"] = (0.2 * rng.standard_normal(shape)).astype(np.float32) if bias else None
    return out


def normed(x, kind, eps, gain, bias):
    """The values and what an error of them is measured by, [N, H, d]."""
    y = oc.head_norm(x, kind, eps, gain, bias)
    c = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    r = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    size = r * np.abs(x).mean(-1, keepdims=True) * np.abs(1.0 if gain is None else gain) * np.ones_like(x)
    return y, np.abs(y) + 2 * np.abs(0.0 if bias is None else bias) + size


def rotated_size(size, interleaved):
    d = size.shape[-1]
    i = np.arange(d // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
    out = np.empty_like(size)
    out[..., a] = out[..., b] = size[..., a] + size[..., b]
    return out


def one(ssd, seed, B, N, Hq, Hkv, d, block, cache, new, kind, per_head, bias, inter=False, gain=True,
        eps=1e-6, mean=0.0, std=1.0):
    rng = np.random.default_rng(seed)
    pool = Pool(rng, B, block, Hkv, d, cache, new)
    qkv = bf16(rng, (B, N, Hq + 2 * Hkv, d), std) + mean
    qkv = qkv.to(torch.bfloat16)
    norm = make_norm(rng, Hq, Hkv, d, per_head, bias, gain)
    dev = qkv.cuda()
    q, k, v = dev.split([Hq, Hkv, Hkv], 2)
    pos = rng.integers(0, 700, (B, N, 3))
    freq = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    sec = (d // 4, d // 8, d // 8)
    table = torch.empty((700, d // 2, 2), device="cuda")
    ssd.ssd_rotary_table(700, d // 2, torch.from_numpy(freq).cuda(), table)
    held = {n: None if x is None else torch.from_numpy(x).cuda() for n, x in norm.items()}
    hn = ssd.head_norm(kind, eps, held["q_gain"], held["q_bias"], held["k_gain"], held["k_bias"])
    out = torch.full((B, N, Hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (pool.cache(ssd), ssd.rotary(table, sec, inter), hn, B, N, Hq, i32(new),
            torch.from_numpy(pool.slots(cache, new, N)).cuda(), i32(pos), q, q.stride(1), k,
            k.stride(1), v, v.stride(1), out, st)
    ssd.ssd_cache_append_norm(*args)
    torch.cuda.synchronize()
    assert st.item() == 0
    x = qkv.double().numpy()
    got = out.double().cpu().numpy()
    scale = pool.dscale["k"].cpu().numpy().astype(np.float64)
    codes = oc.TABLE[pool.dev["k"].cpu().numpy()]
    for b in range(B):
        n, c = int(new[b]), int(cache[b])
        y, size = normed(x[b, :, :Hq], kind, eps, norm["q_gain"], norm["q_bias"])
        want, err = oc.rotate(y, pos[b], freq, sec, inter), 2.0 ** -18 * rotated_size(size, inter)
        assert (np.abs(got[b] - want) <= 2.0 ** -8 * np.abs(want) + 2 * err)[:n].all(), b
        assert (got[b, n:] == 9.0).all()
        y, size = normed(x[b, :, Hq:Hq + Hkv], kind, eps, norm["k_gain"], norm["k_bias"])
        want, err = oc.rotate(y, pos[b], freq, sec, inter), 2.0 ** -18 * rotated_size(size, inter)
        for i in range(c // block, -(-(c + n) // block) if n else 0):
            blk = pool.table[b, i]
            lo, hi = max(c, i * block), min(c + n, (i + 1) * block)
            first, end = lo - i * block, hi - i * block
            for g in range(Hkv):
                old_scale = float(pool.scale["k"][blk, g])
                w, s = oc.append_block(oc.TABLE[pool.codes["k"][blk, g]], old_scale, first,
                                       want[lo - c:hi - c, g])
                e = err[lo - c:hi - c, g]
                assert abs(scale[blk, g] - s) <= 2.0 ** -22 * s + e.max() / 448, (b, i, g)
                have, w = codes[blk, g, :end], w[:end]
                tol = 0.5 * oc.e4m3_step(w) * (1 + 2.0 ** -20) + np.abs(w) * 2.0 ** -16
                tol[first:] += e / s
                assert (np.abs(have - w) <= tol).all(), (b, i, g)
    check_blocks(pool, pool.codes["v"], pool.scale["v"], "v", x[:, :, Hq + Hkv:], cache, new)
    return pool, got


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("per_head,bias", [(False, False), (True, True)])
@pytest.mark.parametrize("inter", [False, True])
def test_blocks(ssd, kind, d, per_head, bias, inter):
    cache = [0, 5, 31, 32, 103, 40]
    new = [67, 1, 1, 32, 25, 0]
    one(ssd, d, 6, 67, 6, 2, d, 32, cache, new, kind, per_head, bias, inter)


@pytest.mark.parametrize("Hq,Hkv,N,block", [(1, 1, 1, 16), (8, 8, 1, 128), (32, 8, 3, 64), (5, 5, 33, 16),
                                            (12, 4, 130, 128)])
@pytest.mark.parametrize("per_head", [False, True])
def test_heads(ssd, Hq, Hkv, N, block, per_head):
    rng = np.random.default_rng(N)
    cache, new = rng.integers(0, 100, 4), rng.integers(1, N + 1, 4)
    new[0] = N
    one(ssd, N, 4, N, Hq, Hkv, 64, block, cache, new, "rms", per_head, False)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_no_gains_far_means_and_small_heads(ssd, kind):
    one(ssd, 1, 2, 9, 4, 2, 128, 16, [3, 14], [9, 4], kind, False, False, gain=False)
    one(ssd, 2, 2, 9, 4, 2, 128, 16, [0, 16], [9, 4], kind, True, True, mean=100.0)
    one(ssd, 3, 2, 9, 4, 2, 64, 16, [0, 16], [9, 4], kind, False, True, std=1e-5, eps=1e-3)
    one(ssd, 4, 2, 9, 4, 2, 64, 16, [0, 16], [9, 4], kind, False, True, std=1e15)


def test_without_norm_as_before(ssd):
    """Gains of 1 of unit-norm rows apart, the append without a norm is another call."""
    rng = np.random.default_rng(4)
    outs = []
    for norm in (None, ssd.head_norm("rms", 1e-6)):
        rng = np.random.default_rng(4)
        pool = Pool(rng, 1, 16, 2, 64, [4], [6])
        x = bf16(rng, (1, 6, 2, 64)).cuda()
        table = torch.ones((3, 32, 2), device="cuda")
        out = torch.zeros((1, 6, 2, 64), dtype=torch.bfloat16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = (1, 6, 2, i32([6]), torch.from_numpy(pool.slots([4], [6], 6)).cuda(),
                torch.zeros((1, 6, 3), dtype=torch.int32, device="cuda"), x, 128, x, 128, x, 128, out, st)
        if norm is None:
            ssd.ssd_cache_append(pool.cache(ssd), ssd.rotary(table, (16, 8, 8)), *args)
        else:
            ssd.ssd_cache_append_norm(pool.cache(ssd), ssd.rotary(table, (16, 8, 8)), norm, *args)
        torch.cuda.synchronize()
        assert st.item() == 0
        outs.append((out, pool.dev["v"], pool.dscale["v"]))
    assert torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][2], outs[1][2])
    assert not torch.equal(outs[0][0], outs[1][0])


def test_zeros_and_nan(ssd):
    """A head of zeros gives the bias; a NaN makes its own head NaN and no other."""
    pool = Pool(np.random.default_rng(5), 1, 16, 2, 64, [0], [3])
    x = torch.ones((1, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 0] = 0.0
    x[0, 1, 1, 5] = float("nan")
    bias = torch.full((64,), 0.5, device="cuda")
    table = torch.zeros((1, 32, 2), device="cuda")
    table[..., 0] = 1.0
    out = torch.zeros_like(x)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ssd.ssd_cache_append_norm(pool.cache(ssd), ssd.rotary(table, (32, 0, 0)),
                              ssd.head_norm("rms", 1e-6, None, bias, None, bias), 1, 3, 2, i32([3]),
                              torch.from_numpy(pool.slots([0], [3], 3)).cuda(),
                              torch.zeros((1, 3, 3), dtype=torch.int32, device="cuda"), x, 128, x, 128,
                              x, 128, out, st)
    torch.cuda.synchronize()
    assert st.item() == 0
    assert (out[0, 0] == 0.5).all() and (out[0, 2] == 1.5).all() and (out[0, 1, 0] == 1.5).all()
    assert torch.isnan(out[0, 1, 1]).all()
    k = oc.TABLE[pool.dev["k"].cpu().numpy()][pool.table[0, 0]]
    s = pool.dscale["k"].cpu().numpy()[pool.table[0, 0]]
    assert np.isnan(k[1, 1]).all() and np.allclose(k[:, 2] * s[:, None], 1.5, rtol=1e-6)
    assert np.allclose(k[:, 0] * s[:, None], 0.5, rtol=2.0 ** -4)
