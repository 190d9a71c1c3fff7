"""The operators of a decoding pass over the paged 8-bit cache, as a program calls them.

A program that decodes images token by token, or verifies drafts, over a cache that
is paged and held in 8 bits runs per pass: the plan (which blocks and slots the new
tokens take), the append (rotary positions with three axes, quantised write), the
attention over the blocks and the sampler.  Kinds of case:

  plan    ssd_cache_plan: block tables, slot maps and positions from request lengths
  append  ssd_cache_append: q and k rotated, k and v written as e4m3 with a scale for
          each block and head
  attn    ssd_cache_attention: frontier attention over the blocks
  sample  ssd_sample: temperature, top-k, top-p, min-p with given uniforms

Sizes are those of the repository's workloads (16x16, 24x24, 32x32 and 64x64 grids, 8 x 64
to 32 x 128 heads, vocabularies of 4096 to 65536) and generic ones: one token for each of
many requests, prompts of a thousand tokens, caches of 32768.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TOP = 448.0           # largest e4m3 value
FLOOR = 2.0 ** -100   # least amax a block is scaled by
LOG2E = 1.4426950408889634


# ------------------------------------------------------------------------ cases
def listed():
    return [
        # smallest: sixteen images, one new token each, of which a few open a block
        dict(name="plan_token_b16", op="plan", H=24, W=24, prefix=120, B=16, N=1, block=64,
             len_lo=120, len_hi=696, lens=1),
        # a batch of prompts and partly generated images admitted at once
        dict(name="plan_prompts_b256", op="plan", H=32, W=32, prefix=64, B=256, N=1088, block=16,
             len_lo=0, len_hi=0, lens=2),
        # one token of each of eight images, into blocks that are partly full: latency counts
        dict(name="append_token_b8", op="append", H=32, W=32, prefix=64, B=8, N=1, Hq=32, Hkv=8,
             d=128, block=64, len_lo=64, len_hi=1088, lens=3, interleaved=False, fused=True),
        # the drafted rows of the 64x64 batch, whole heads
        dict(name="append_64x64_b8", op="append", H=64, W=64, prefix=256, B=8, N=128, Hq=32,
             Hkv=32, d=128, block=64, len_lo=256, len_hi=4224, lens=4, interleaved=False,
             fused=False),
        # ragged prompts and images to be continued, up to 1088 tokens, grouped heads
        dict(name="append_prompts_b16", op="append", H=32, W=32, prefix=64, B=16, N=1088, Hq=32,
             Hkv=8, d=128, block=32, len_lo=0, len_hi=0, lens=5, interleaved=True, fused=True),
        # smallest attention: one 16x16 image's two rows, 64-wide heads
        dict(name="attn_16x16_b1", op="attn", H=16, W=16, prefix=32, B=1, N=32, full=True, Hq=8,
             Hkv=8, d=64, block=16, len_lo=192, len_hi=192, lens=6),
        # plain decoding of long sequences: one token each, grouped heads, ragged to 32768
        dict(name="attn_token_b16_long", op="attn", H=180, W=180, prefix=256, B=16, N=1, full=True,
             Hq=32, Hkv=8, d=128, block=64, len_lo=6000, len_hi=32600, lens=7),
        # 24x24 images at all stages, two drafted rows each
        dict(name="attn_24x24_b25", op="attn", H=24, W=24, prefix=120, B=25, N=48, full=True,
             Hq=16, Hkv=16, d=128, block=32, len_lo=120, len_hi=648, lens=8),
        # the 64x64 batch past its middle, two drafted rows each
        dict(name="attn_64x64_b8", op="attn", H=64, W=64, prefix=256, B=8, N=128, full=True,
             Hq=32, Hkv=32, d=128, block=64, len_lo=2300, len_hi=3801, lens=9),
        # the sampler of one image: top 2000 of 16384
        dict(name="sample_b1", op="sample", rows=1, V=16384, bf16=False, logits="normal",
             temperature=1.0, top_k=2000, top_p=1.0, min_p=0.0, per_row=False),
        # every drafted row of the 64x64 batch, nucleus of the whole vocabulary
        dict(name="sample_1024_p95", op="sample", rows=1024, V=65536, bf16=False, logits="zipf",
             temperature=1.0, top_k=0, top_p=0.95, min_p=0.0, per_row=False),
        # requests with settings of their own, bf16 logits of an odd vocabulary
        dict(name="sample_200_mixed", op="sample", rows=200, V=32771, bf16=True, logits="normal",
             temperature=0.9, top_k=500, top_p=0.9, min_p=0.002, per_row=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["plan", "append", "append", "attn", "attn", "attn", "sample", "sample"])
    if op == "sample":
        return dict(op=op, rows=_log_int(rng, 1, 1024), V=_log_int(rng, 1000, 65536),
                    bf16=rng.random() < 0.4, logits=rng.choice(["normal", "zipf"]),
                    temperature=round(rng.uniform(0.5, 1.5), 3),
                    top_k=rng.choice([0, 1, _log_int(rng, 2, 4000), _log_int(rng, 2, 4000)]),
                    top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                    min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.0005, 0.1), 4)]),
                    per_row=rng.random() < 0.4)
    W = rng.choice([16, 24, 32, 48, 64, rng.randrange(16, 65)])
    prefix = rng.randrange(16, 257)
    full = prefix + W * W
    block = rng.choice([16, 32, 64, 64, 128])
    B = _log_int(rng, 1, 32)
    c = dict(op=op, H=W, W=W, prefix=prefix, B=B, block=block, lens=rng.randrange(1 << 20))
    N = rng.choice([1, _log_int(rng, 1, 128), _log_int(rng, 1, 128)])
    if op == "plan":
        c.update(B=_log_int(rng, 1, 256), N=_log_int(rng, 1, 1088))
        c["N"] = min(c["N"], full)
        c["len_hi"] = rng.randrange(0, full - c["N"] + 1)
        c["len_lo"] = rng.randrange(0, c["len_hi"] + 1)
        return c
    heads = [(8, 8, 64), (16, 16, 128), (32, 8, 128), (32, 32, 128), (12, 4, 64), (6, 2, 128)]
    Hq, Hkv, d = rng.choice(heads)
    if op == "append":
        N = min(rng.choice([N, N, _log_int(rng, 64, 1088)]), full)
        c.update(N=N, Hq=Hq, Hkv=Hkv, d=d, len_hi=rng.randrange(0, full - N + 1),
                 interleaved=rng.random() < 0.5, fused=rng.random() < 0.5)
        c["len_lo"] = rng.randrange(0, c["len_hi"] + 1)
        return c
    if N == 1 and rng.random() < 0.5:  # long sequences, token by token
        c.update(H=180, W=180)
        full = prefix + 180 * 180
    c["N"], c["full"] = min(N, full), rng.random() < 0.6
    c.update(Hq=Hq, Hkv=Hkv, d=d, len_hi=_log_int(rng, 64, full - c["N"]))
    c["len_lo"] = rng.randrange(0, c["len_hi"] + 1)
    return c


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op)
            for op in ("plan", "append", "attn", "sample")}
    while True:
        c = _draw(rng)
        if _cost(c) <= most[c["op"]]:
            return c
        c["rows" if c["op"] == "sample" else "B"] //= 2
        if c.get("rows", c.get("B")) and _cost(c) <= most[c["op"]]:
            return c


def _lengths(case):
    """Cache length and new tokens of every request."""
    r = random.Random(case["lens"])
    B, N = case["B"], case["N"]
    cache = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(B)]
    new = [N if case.get("full") or r.random() < 0.25 else r.randint((N + 7) // 8, N)
           for _ in range(B)]
    if B > 2 and not case.get("full"):
        new[r.randrange(B)] = 0  # a request that has nothing new
    return cache, new


def _blocks(n, block):
    return -(-n // block)


def _demand(case):
    cache, new = _lengths(case)
    S = case["block"]
    return [_blocks(c + n, S) - _blocks(c, S) for c, n in zip(cache, new)]


def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["V"]
        return dict(bytes=n * (2 if case["bf16"] else 4) + case["rows"] * 20, flops=4 * n)
    cache, new = _lengths(case)
    B, N, T = case["B"], case["N"], sum(new)
    if case["op"] == "plan":
        return dict(bytes=16 * B + 8 * sum(_demand(case)) + 20 * B * N, flops=0)
    Hq, Hkv, d, S = case["Hq"], case["Hkv"], case["d"], case["block"]
    if case["op"] == "append":
        touched = sum(_blocks(c + n, S) - c // S for c, n in zip(cache, new) if n)
        return dict(bytes=T * (Hq + 2 * Hkv) * d * 2 + 20 * T + T * Hq * d * 2 + T * 2 * Hkv * d
                    + touched * Hkv * 8, flops=3 * T * (Hq + Hkv) * d + 4 * T * Hkv * d)
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cache, new))
    keys = sum(c + n for c, n in zip(cache, new) if n)
    return dict(bytes=keys * Hkv * 2 * d + 8 * Hkv * (keys // S) + 2 * T * Hq * d * 2,
                flops=4 * d * Hq * pairs)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


# ---------------------------------------------------------------------- prepare
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _table(case, gen):
    """A block table over a pool in random order: rows of the blocks that hold the cached
    and the new tokens, -1 behind them."""
    cache, new = _lengths(case)
    S, B = case["block"], case["B"]
    need = [_blocks(c + n, S) for c, n in zip(cache, new)]
    pool = sum(need) + 3
    ids = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
    M = max(max(need), 1)
    first = np.concatenate([[0], np.cumsum(need)])[:-1]
    at = torch.from_numpy(first).to(DEV)[:, None] + torch.arange(M, device=DEV)[None]
    have = torch.arange(M, device=DEV)[None] < _i32(need)[:, None]
    table = torch.where(have, ids[at.clamp(max=pool - 1)], -1).to(torch.int32).contiguous()
    return table, pool


def _slots(case, table):
    cache, new = _lengths(case)
    S, N = case["block"], case["N"]
    p = _i32(cache).long()[:, None] + torch.arange(N, device=DEV)[None]
    blk = torch.gather(table.long(), 1, (p // S).clamp(max=table.shape[1] - 1))
    live = torch.arange(N, device=DEV)[None] < _i32(new)[:, None]
    return torch.where(live, blk * S + p % S, -1).contiguous()


def _positions(case):
    cache, _ = _lengths(case)
    P, W, N = case["prefix"], case["W"], case["N"]
    p = _i32(cache).long()[:, None] + torch.arange(N, device=DEV)[None]
    i = (p - P).clamp(min=0)
    text = p < P
    pos = torch.stack([torch.where(text, p, P), torch.where(text, p, P + i // W),
                       torch.where(text, p, P + i % W)], -1)
    return pos.to(torch.int32).contiguous()


def _values(gen, shape, dtype):
    """Projections as layers give them: normal, heads of unequal size, a few wide channels."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x *= torch.exp(0.3 * torch.randn((shape[-2], 1), generator=gen, device=DEV))
    wide = torch.rand(shape[-1], generator=gen, device=DEV) < 0.03
    return (x * torch.where(wide, 3.0, 1.0)).to(dtype)


def _fill(gen, pool, Hkv, S, d):
    """A cache that earlier tokens filled: values within their scales."""
    scale = 0.004 * torch.exp(0.3 * torch.randn((pool, Hkv), generator=gen, device=DEV))
    x = torch.randn((pool, Hkv, S, d), generator=gen, device=DEV)
    return (x / scale[:, :, None, None]).clamp(-TOP, TOP).to(E4M3), scale.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1000003 + 17)
    s = dict(case=dict(case), status=torch.zeros(1, dtype=torch.int32, device=DEV))
    if case["op"] == "sample":
        rows, V = case["rows"], case["V"]
        if case["logits"] == "zipf":
            rank = torch.argsort(torch.rand((rows, V), generator=gen, device=DEV), dim=1)
            x = -1.1 * torch.log(rank.float() + 1.0)
            x += torch.randn((rows, V), generator=gen, device=DEV)
        else:
            x = 2.0 * torch.randn((rows, V), generator=gen, device=DEV)
        s["logits"] = x.to(torch.bfloat16) if case["bf16"] else x
        s["uniforms"] = torch.rand((rows, 2), generator=gen, device=DEV)
        if case["per_row"]:
            r = lambda: torch.rand(rows, generator=gen, device=DEV)  # noqa: E731
            s["temperature"] = (case["temperature"] * (0.8 + 0.4 * r())).contiguous()
            s["temperature"][r() < 0.1] = 0.0  # greedy requests
            s["top_k"] = (case["top_k"] * 2 * r()).to(torch.int32)  # 0: no limit
            s["top_p"] = (1 - (1 - case["top_p"]) * 2 * r()).clamp(0.05, 1.0).contiguous()
            s["min_p"] = (case["min_p"] * 2 * r()).contiguous()
        for name, dt in (("tok", torch.int32), ("prob", torch.float32), ("kept", torch.int32)):
            s[name] = torch.zeros(rows, dtype=dt, device=DEV)
        return s
    cache, new = _lengths(case)
    S, N, B = case["block"], case["N"], case["B"]
    s["cache_len"], s["n_new"] = _i32(cache), _i32(new)
    if case["op"] == "plan":
        held = [_blocks(c, S) for c in cache]
        M = max(_blocks(c + N, S) for c in cache)
        pool = sum(held) + sum(_demand(case)) + 5
        ids = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
        s["held"], s["pool"], s["M"] = _i32(held), pool, M
        first = torch.cumsum(s["held"], 0) - s["held"]
        at = first[:, None] + torch.arange(M, device=DEV)[None]
        mine = torch.arange(M, device=DEV)[None] < s["held"][:, None]
        s["table"] = torch.where(mine, ids[at.clamp(max=pool - 1)], -1).to(torch.int32).contiguous()
        s["ring"] = torch.roll(ids, -sum(held)).contiguous()  # the free ones first
        head = 7 * pool + pool // 2  # blocks dealt so far: the ring has turned seven times
        s["head"] = torch.tensor([head], dtype=torch.int64, device=DEV)
        s["tail"] = s["head"] + (pool - sum(held))
        s["ring"] = torch.roll(s["ring"], head % pool).contiguous()
        s["next_head"] = torch.zeros_like(s["head"])
        s["n_blocks"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        s["slots"] = torch.zeros((B, N), dtype=torch.int64, device=DEV)
        s["pos"] = torch.zeros((B, N, 3), dtype=torch.int32, device=DEV)
        return s
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    s["table"], s["pool"] = _table(case, gen)
    s["k"], s["k_scale"] = _fill(gen, s["pool"], Hkv, S, d)
    s["v"], s["v_scale"] = _fill(gen, s["pool"], Hkv, S, d)
    if case["op"] == "attn":
        q = _values(gen, (B, N, Hq, d), torch.float32)
        s["q"] = (1.5 * q).to(torch.bfloat16)
        s["o"] = torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device=DEV)
        return s
    s["slots"], s["pos"] = _slots(case, s["table"]), _positions(case)
    # rotary table: a quarter of the pairs by time, the rest by row and column
    pairs = d // 2
    s["sections"] = (pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8)
    freq = 10000.0 ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / pairs)
    angle = torch.arange(case["prefix"] + case["H"] * case["W"] + 1, device=DEV,
                         dtype=torch.float64)[:, None] * freq.float().double()[None]
    s["rotary"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
    if case["fused"]:  # one buffer, as a joint projection writes it
        qkv = _values(gen, (B, N, Hq + 2 * Hkv, d), torch.bfloat16)
        s["new_q"], s["new_k"], s["new_v"] = qkv.split([Hq, Hkv, Hkv], 2)
    else:
        s["new_q"] = _values(gen, (B, N, Hq, d), torch.bfloat16)
        s["new_k"] = _values(gen, (B, N, Hkv, d), torch.bfloat16)
        s["new_v"] = _values(gen, (B, N, Hkv, d), torch.bfloat16)
    s["q_out"] = torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device=DEV)
    return s


# -------------------------------------------------------------------------- run
def run(s):
    return globals()[("own_" if own else "plain_") + s["case"]["op"]](s)


def own_plan(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    if "grid" not in s:
        s["grid"] = ssd.grid(c["H"], c["W"], c["prefix"])
    ssd.ssd_cache_plan(s["grid"], c["B"], c["block"], s["M"], c["N"], s["cache_len"], s["n_new"],
                       s["held"], s["ring"], s["pool"], s["head"], s["tail"], s["next_head"],
                       s["table"], s["n_blocks"], s["slots"], s["pos"], s["status"])
    return dict(table=s["table"], n_blocks=s["n_blocks"], next_head=s["next_head"],
                slots=s["slots"], pos=s["pos"], status=s["status"])


def plain_plan(s):
    c = s["case"]
    S, N, M = c["block"], c["N"], s["M"]
    end = s["cache_len"] + s["n_new"]
    need = (end + S - 1) // S
    demand = (need - s["held"]).clamp(min=0)
    stop = torch.cumsum(demand.long(), 0)
    first = stop - demand
    served = s["head"] + stop <= s["tail"]
    i = torch.arange(M, device=DEV)[None] - s["held"][:, None]
    fresh = (i >= 0) & (i < demand[:, None]) & served[:, None]
    ids = s["ring"][((s["head"] + first)[:, None] + i.clamp(min=0)) % s["pool"]]
    table = torch.where(fresh, ids, s["table"])
    n_blocks = torch.where(served, torch.maximum(need, s["held"]), s["held"]).to(torch.int32)
    p = s["cache_len"].long()[:, None] + torch.arange(N, device=DEV)[None]
    live = (torch.arange(N, device=DEV)[None] < s["n_new"][:, None]) & served[:, None]
    block = torch.gather(table.long(), 1, (p // S).clamp(max=M - 1))
    slots = torch.where(live, block * S + p % S, -1)
    pre, W = c["prefix"], c["W"]
    g = (p - pre).clamp(min=0)
    pos = torch.stack([p.clamp(max=pre), torch.where(p < pre, p, pre + g // W),
                       torch.where(p < pre, p, pre + g % W)], -1)
    pos = torch.where(live[:, :, None], pos, 0).to(torch.int32)
    taken = torch.where(served, stop, 0).max()
    return dict(table=table, n_blocks=n_blocks, next_head=s["head"] + taken, slots=slots, pos=pos,
                status=s["status"])


def _own_cache(s, ssd):
    if "cache" not in s:
        s["cache"] = ssd.cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    return s["cache"]


def own_append(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    if "rot" not in s:
        s["rot"] = ssd.rotary(s["rotary"], s["sections"], c["interleaved"])
    ssd.ssd_cache_append(_own_cache(s, ssd), s["rot"], c["B"], c["N"], c["Hq"], s["n_new"],
                         s["slots"], s["pos"], s["new_q"], s["new_q"].stride(1), s["new_k"],
                         s["new_k"].stride(1), s["new_v"], s["new_v"].stride(1), s["q_out"],
                         s["status"])
    return dict(q=s["q_out"], k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                status=s["status"])


def _rotate(s, x):
    c = s["case"]
    sec = s["sections"]
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(sec, device=DEV))
    rows = s["pos"].long()[:, :, axis]
    cs = s["rotary"][rows, torch.arange(sum(sec), device=DEV)]
    cos, sin = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
    x = x.float()
    if c["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _write(s, x, cache, scale):
    """x [B, N, Hkv, d] into the cache at the slots: the new cache and its scales."""
    S = s["case"]["block"]
    pool, Hkv = scale.shape
    live = s["slots"] >= 0
    slot = s["slots"][live]
    blk, off, x = slot // S, slot % S, x[live]
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m = torch.zeros_like(scale).scatter_reduce(0, blk[:, None].expand(-1, Hkv), amax, "amax")
    first = torch.full((pool,), S, device=DEV).scatter_reduce(0, blk, off, "amin")[:, None]
    touched = first < S
    kept = touched & (first > 0)
    old_top = TOP * scale
    grown = touched & (~kept | (m > old_top))
    new_scale = torch.where(grown, m.clamp(min=FLOOR) / TOP, scale)
    inv = 1.0 / new_scale
    factor = (scale * inv)[:, :, None, None]
    again = (kept & grown)[:, :, None, None] & (torch.arange(S, device=DEV)[:, None]
                                                < first[:, :, None, None])
    cache = torch.where(again, (cache.float() * factor).to(E4M3).float(), cache.float())
    cache[blk, :, off] = (x * inv[blk][:, :, None]).clamp(-TOP, TOP).to(E4M3).float()
    return cache.to(E4M3), new_scale


def plain_append(s):
    q = _rotate(s, s["new_q"]).to(torch.bfloat16)
    q = torch.where((s["slots"] >= 0)[:, :, None, None], q, 0)
    k, ks = _write(s, _rotate(s, s["new_k"]), s["k"], s["k_scale"])
    v, vs = _write(s, s["new_v"].float(), s["v"], s["v_scale"])
    return dict(q=q, k=k, v=v, k_scale=ks, v_scale=vs, status=s["status"])


def own_attn(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    if "grid" not in s:
        s["grid"] = ssd.grid(c["H"], c["W"], c["prefix"])
        n = ssd.ssd_cache_attention_workspace(c["B"], c["Hq"], c["Hkv"], c["d"], c["N"],
                                              s["table"].shape[1] * c["block"])
        s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    ssd.ssd_cache_attention(s["grid"], _own_cache(s, ssd), c["B"], c["Hq"], s["cache_len"],
                            s["n_new"], None, None, c["N"], s["table"], s["table"].shape[1], s["q"],
                            0.0, s["o"], None, s["ws"], s["ws"].numel(), s["status"])
    return dict(o=s["o"], status=s["status"])


def plain_attn(s):
    c = s["case"]
    B, N, Hq, Hkv, d, S = c["B"], c["N"], c["Hq"], c["Hkv"], c["d"], c["block"]
    L, G = s["table"].shape[1] * S, Hq // Hkv

    def gathered(x, scale):
        at = s["table"].long().clamp(min=0)
        y = x[at].float() * scale[at][:, :, :, None, None]          # [B, M, Hkv, S, d]
        return y.transpose(1, 2).reshape(B, Hkv, L, d)

    at = torch.arange(L, device=DEV)[None]
    end = s["cache_len"] + s["n_new"]
    k = torch.where((at < end[:, None])[:, None, :, None], gathered(s["k"], s["k_scale"]), 0.0)
    q = s["q"].float().reshape(B, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, d)
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    del k
    row = torch.arange(N, device=DEV)[None]
    seen = (at[:, None] <= (s["cache_len"][:, None] + row)[:, :, None])   # [B, N, L]
    seen = seen & (row < s["n_new"][:, None])[:, :, None]
    seen = seen.repeat_interleave(G, 1)[:, None]
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp_(x.sub_(torch.where(torch.isfinite(top), top, 0.0)))
    x /= x.sum(-1, keepdim=True).clamp(min=1e-30)
    v = torch.where((at < end[:, None])[:, None, :, None], gathered(s["v"], s["v_scale"]), 0.0)
    o = torch.matmul(x, v).reshape(B, Hkv, N, G, d).permute(0, 2, 1, 3, 4)
    return dict(o=o.reshape(B, N, Hq, d).to(torch.bfloat16), status=s["status"])


def own_sample(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    if "how" not in s:
        s["rng"] = ssd.rng(uniforms=s["uniforms"])
        s["how"] = ssd.sampling(c["temperature"], c["top_k"], c["top_p"], c["min_p"],
                                *([s["temperature"], s["top_k"], s["top_p"], s["min_p"]]
                                  if c["per_row"] else []))
    ssd.ssd_sample(c["rows"], c["V"], s["logits"], c["V"], s["how"], s["rng"], s["tok"], s["prob"],
                   s["kept"], s["status"])
    return dict(tok=s["tok"], prob=s["prob"], kept=s["kept"], status=s["status"])


def _settings(s):
    c = s["case"]
    if c["per_row"]:
        return s["temperature"], s["top_k"], s["top_p"], s["min_p"]
    one = lambda v, dt: torch.full((c["rows"],), v, dtype=dt, device=DEV)  # noqa: E731
    return (one(c["temperature"], torch.float32), one(c["top_k"], torch.int32),
            one(c["top_p"], torch.float32), one(c["min_p"], torch.float32))


def plain_sample(s):
    V = s["case"]["V"]
    T, k, p, mp = _settings(s)
    k = torch.where(T > 0, torch.where((k <= 0) | (k > V), V, k), 1)[:, None]
    x = s["logits"].float()
    top = x.amax(-1, keepdim=True)
    c = torch.where(T > 0, torch.full_like(T, LOG2E) / torch.where(T > 0, T, 1.0), 1.0)[:, None]
    w = torch.exp2(-((top - x) * c))
    W = torch.round(w * 2.0 ** 31).long()
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    Ws = torch.gather(W, 1, order)
    Ws = torch.where(torch.arange(V, device=DEV)[None] < k, Ws, 0)
    total = Ws.sum(-1, keepdim=True)
    before = torch.cumsum(Ws, -1) - Ws
    ok = (Ws > 0) & (before.double() < p.double()[:, None] * total.double())
    ok &= torch.gather(w, 1, order) >= mp[:, None]
    kept = torch.zeros_like(ok).scatter(1, order, ok)
    cum = torch.cumsum(torch.where(kept, W, 0), -1)
    Z = cum[:, -1:]
    aim = s["uniforms"][:, 1:].double() * Z.double()
    tok = (cum.double() <= aim).sum(-1, keepdim=True)
    prob = (torch.gather(W, 1, tok).double() / Z.double()).float()
    return dict(tok=tok[:, 0].to(torch.int32), prob=prob[:, 0], kept=ok.sum(-1).to(torch.int32),
                status=s["status"])


# ------------------------------------------------------------------------ exact
def exact(case, seed):
    s = prepare(case, seed)
    return globals()["exact_" + case["op"]](s)


def exact_plan(s):
    return None  # whole numbers only


def _round8(x):
    """The nearest e4m3 value, ties to even, in 64 bits."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6.0)
    step = torch.exp2(e - 3.0)
    return (torch.round(x / step) * step).clamp(-TOP, TOP)


def exact_append(s):
    """Token by token for the positions, block by block for the scales."""
    c = s["case"]
    S, d, Hkv = c["block"], c["d"], c["Hkv"]
    cache_len, new = _lengths(c)
    sec, pairs = s["sections"], d // 2
    axis = [0] * sec[0] + [1] * sec[1] + [2] * sec[2]
    freq = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], dtype=torch.float64,
                        device=DEV).float().double()
    t = s["pos"][:, :, axis].double() * freq
    z = torch.polar(torch.ones_like(t), t)[:, :, None]

    def turned(x):
        x = x.double()
        a, b = (x[..., 0::2], x[..., 1::2]) if c["interleaved"] else (x[..., :pairs], x[..., pairs:])
        y = torch.complex(a, b) * z
        return (torch.stack([y.real, y.imag], -1).flatten(-2) if c["interleaved"]
                else torch.cat([y.real, y.imag], -1))

    q = turned(s["new_q"])
    out = dict(q=q, status=None)
    for name, x in (("k", turned(s["new_k"])), ("v", s["new_v"].double())):
        cache, scale = s[name].double(), s[name + "_scale"].double()
        for b, (at, n) in enumerate(zip(cache_len, new)):
            q[b, n:] = 0
            for i in range(at // S, _blocks(at + n, S) if n else 0):
                blk = int(s["table"][b, i])
                lo, hi = max(at, i * S), min(at + n, (i + 1) * S)
                old = lo - i * S
                y = x[b, lo - at:hi - at].transpose(0, 1)               # [Hkv, n, d]
                m = y.abs().amax((1, 2))
                grown = (m > TOP * scale[blk]) if old else torch.ones_like(m, dtype=torch.bool)
                fresh = torch.where(grown, m.clamp(min=FLOOR) / TOP, scale[blk])
                r = (scale[blk] / fresh)[:, None, None]
                again = _round8(cache[blk, :, :old] * r)
                cache[blk, :, :old] = torch.where(grown[:, None, None], again, cache[blk, :, :old])
                cache[blk, :, old:old + hi - lo] = _round8(y / fresh[:, None, None])
                scale[blk] = fresh
        out[name], out[name + "_scale"] = cache, scale
    return out


def exact_attn(s):
    c = s["case"]
    G, d = c["Hq"] // c["Hkv"], c["d"]
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV)
    for b, (at, n) in enumerate(zip(*_lengths(c))):
        blocks = s["table"][b, :_blocks(at + n, c["block"])].long()
        for g in range(c["Hkv"]):
            k, v = ((s[x][blocks, g].double() * s[x + "_scale"][blocks, g].double()[:, None, None])
                    .reshape(-1, d)[:at + n] for x in ("k", "v"))
            x = torch.einsum("nhd,sd->nhs", s["q"][b, :n, g * G:(g + 1) * G].double(), k)
            hide = torch.ones((n, at + n), dtype=torch.bool, device=DEV).triu(at + 1)
            p = torch.softmax((x / math.sqrt(d)).masked_fill(hide[:, None], -math.inf), -1)
            o[b, :n, g * G:(g + 1) * G] = torch.einsum("nhs,sd->nhd", p, v)
    return dict(o=o, status=None)


def exact_sample(s):
    """One row after the other on the host, the weights as they are."""
    c = s["case"]
    x = s["logits"].double().cpu().numpy()
    T, k, p, mp = (v.double().cpu().numpy() for v in _settings(s))
    u = s["uniforms"].double().cpu().numpy()[:, 1]
    prob = np.zeros(c["rows"])
    for r in range(c["rows"]):
        if T[r] == 0:
            prob[r] = 1.0
            continue
        order = np.argsort(-x[r], kind="stable")
        if 0 < k[r] < c["V"]:
            order = order[:int(k[r])]
        w = np.exp((x[r][order] - x[r][order[0]]) / T[r])
        n = int(np.searchsorted(np.cumsum(w), p[r] * w.sum())) + 1
        n = min(n, int((w >= mp[r]).sum()), len(w))
        ids = np.sort(order[:n])
        w = np.exp((x[r][ids] - x[r].max()) / T[r])
        at = min(int(np.searchsorted(np.cumsum(w), u[r] * w.sum(), side="right")), n - 1)
        prob[r] = w[at] / w.sum()
    return dict(tok=None, prob=torch.from_numpy(prob), kept=None, status=None)
