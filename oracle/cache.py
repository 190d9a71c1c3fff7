"""The paged 8-bit cache in float64: e4m3, the plan, the append and the
attention over the blocks, from their definitions (include/ssd.h), one
sequence, block and head after the other.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

TOP = 448.0
LEAST = 2.0 ** -100


def e4m3_table() -> np.ndarray:
    """The 256 values of e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits;
    all exponent and mantissa bits set is NaN, there is no infinity."""
    out = np.empty(256)
    for i in range(256):
        e, m = (i >> 3) & 15, i & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            x = np.nan
        out[i] = -x if i >> 7 else x
    return out


TABLE = e4m3_table()


def e4m3_step(x):
    """Distance of the e4m3 values around |x|."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    return 2.0 ** (np.minimum(e, 8) - 3)


def e4m3_round(x):
    """Nearest e4m3 value, ties to even, +-448 beyond; NaN stays."""
    s = e4m3_step(x)
    r = np.rint(x / s) * s
    return np.where(np.isnan(x), np.nan, np.clip(r, -TOP, TOP))


def plan(grid_w, row_stride, prefix, block, max_blocks, N, cache_len, n_new, held, ring, head, tail,
         table):
    """(table, n_blocks, next_head, slots, pos, served) as ssd_cache_plan writes them."""
    B, R = len(cache_len), len(ring)
    table = np.array(table, copy=True)
    n_blocks = np.array(held, copy=True)
    slots = np.full((B, N), -1, np.int64)
    pos = np.zeros((B, N, 3), np.int32)
    at = int(head)
    blocked = False
    served = np.zeros(B, bool)
    for b in range(B):
        c, n, h = int(cache_len[b]), int(n_new[b]), int(held[b])
        need = -(-(c + n) // block)
        if c < 0 or n < 0 or n > N or h < 0 or h > max_blocks or need > max_blocks:
            continue
        want = max(0, need - h)
        if want and (blocked or at + want > tail):
            blocked = True
            continue
        served[b] = True
        for i in range(want):
            table[b, h + i] = ring[(at + i) % R]
        at += want
        n_blocks[b] = h + want
        for j in range(n):
            p = c + j
            slots[b, j] = int(table[b, p // block]) * block + p % block
            if p < prefix:
                pos[b, j] = p
            else:
                y, x = divmod(p - prefix, row_stride)
                pos[b, j] = (prefix, prefix + y, prefix + x)
    return table, n_blocks, at, slots, pos, served


def rotate(x, pos, freq, sections, interleaved):
    """x [N, H, d], pos [N, 3]: every pair turned by its axis' position."""
    d = x.shape[-1]
    axis = np.repeat(np.arange(3), sections)
    angle = pos[:, axis].astype(np.float64) * freq.astype(np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    i = np.arange(d // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
    y = np.empty_like(x, dtype=np.float64)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def append_block(old, old_scale, first, new):
    """One block and head: `old` [block, d] the entries it holds (its first
    `first` tokens live), `new` [n, d] values for the tokens from `first` on.
    Returns (what the entries should stand for before rounding [block, d] (NaN:
    not written), the new scale)."""
    fin = np.abs(new[np.isfinite(new)])
    m = fin.max() if fin.size else 0.0
    grown = first == 0 or m > TOP * old_scale
    scale = max(m, LEAST) / TOP if grown else old_scale
    want = np.full(old.shape, np.nan)
    if grown:
        want[:first] = old[:first] * (old_scale / scale)
    else:
        want[:first] = old[:first]
    want[first:first + len(new)] = np.clip(new / scale, -TOP, TOP)
    return want, scale


def attention(q, k, v, visible, scale, vscale):
    """q [n, Hq, d], k, v [L, Hkv, d] float64, visible [n, L], vscale [L, Hkv] the
    scales that v contains.  Returns o, lse and three magnitudes for error bounds: A =
    sum p |v|; F = sum |v| (largest scale / its scale) / sum exp(x - max), what an absolute
    error of the weights amounts to; mag = scale * max |q| * the largest sum |k|."""
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    o, A, F = np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, mag = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for h in range(Hq):
        g = h // G
        for j in range(n):
            see = visible[j]
            if not see.any():
                continue
            kk, vv, vs = k[see, g], v[see, g], vscale[see, g]
            x = kk @ q[j, h] * scale
            m = x.max()
            p = np.exp(x - m)
            z = p.sum()
            o[j, h], A[j, h] = p @ vv / z, p @ np.abs(vv) / z
            F[j, h] = (vs.max() / vs) @ np.abs(vv) / z
            lse[j, h] = m + np.log(z)
            mag[j, h] = np.abs(q[j, h]).max() * np.abs(kk).sum(-1).max() * scale
    return o, lse, A, F, mag


def head_norm(x, kind, eps, gain=None, bias=None):
    """x [N, H, d] float64: every head over its d values; gain, bias [d] or [H, d]."""
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        y = y * gain
    return y if bias is None else y + bias
