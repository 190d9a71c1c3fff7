"""The operators around the paged 8-bit cache that a decoder layer runs, as a program calls them.

A program that decodes images over the paged 8-bit cache, several of them from one prompt,
runs per layer: the projections on 8-bit inputs and weights, the append with the norms of
the query and key heads, and the attention of sequences that share the blocks of their
prompt.  Kinds of case:

  quant   ssd_quantize: rows (or square blocks of a weight) to e4m3, a scale per 128 entries
  matmul  ssd_scaled_matmul: products of such rows and weights, with or without a residual
  norm    ssd_cache_append_norm: head norms, rotation, quantised write into the cache
  shared  ssd_cache_attention_shared: frontier attention, shared blocks read once a group

Sizes are those of the repository's workloads (16x16 to 64x64 grids, 8 x 64 to 32 x 128
heads, widths of 4096 and 8192, vocabularies up to 65536, 8 x 128 drafts, prompts of 1088
tokens) and generic ones: caches of 32768, odd widths.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TOP = 448.0           # largest e4m3 value
FLOOR = 2.0 ** -100   # least amax a scale is taken from
G128 = 128            # entries of a scale


# ------------------------------------------------------------------------ cases
def listed():
    return [
        # the hidden states of one token of each of eight images
        dict(name="quant_token_b8", op="quant", rows=8, K=4096, block_rows=1, bf16=True, gap=0),
        # the hidden states of a batch of prompts
        dict(name="quant_prompts", op="quant", rows=17408, K=4096, block_rows=1, bf16=True, gap=0),
        # one token of eight images through the joint projection of q, k and v
        dict(name="matmul_token_b8", op="matmul", M=8, N=6144, K=4096, bf16=True, add=False, gap=0),
        # logits of sixteen images for the sampler
        dict(name="matmul_head_b16", op="matmul", M=16, N=65536, K=4096, bf16=False, add=False,
             gap=0),
        # an odd width and few rows that are parts of wider ones
        dict(name="matmul_odd_200", op="matmul", M=200, N=5000, K=2050, bf16=True, add=False,
             gap=48),
        # 8 x 128 drafts: the attention's way out, added to the residual stream
        dict(name="matmul_drafts_add", op="matmul", M=1024, N=4096, K=4096, bf16=True, add=True,
             gap=0),
        # a batch of prompts into the wide side of an MLP
        dict(name="matmul_prompts", op="matmul", M=17408, N=12288, K=4096, bf16=True, add=False,
             gap=0),
        # one token of each of eight images, root-mean-square norms with one gain for all heads
        dict(name="norm_token_b8", op="norm", H=32, W=32, prefix=64, B=8, N=1, Hq=32, Hkv=8, d=128,
             block=64, len_lo=64, len_hi=1088, lens=3, interleaved=False, layer=False,
             per_head=False),
        # ragged prompts of up to 1088 tokens, layer norms with gains and biases of every head
        dict(name="norm_prompts_b16", op="norm", H=32, W=32, prefix=64, B=16, N=1088, Hq=32,
             Hkv=8, d=128, block=32, len_lo=0, len_hi=0, lens=5, interleaved=True, layer=True,
             per_head=True),
        # four 16x16 images of one prompt, a token each
        dict(name="shared_16x16_b4", op="shared", B=4, groups=1, N=1, full=True, Hq=8, Hkv=8, d=64,
             block=16, pre_lo=192, pre_hi=192, own_lo=10, own_hi=200, lens=6),
        # sixty-four images of one prompt that holds an image, a token each
        dict(name="shared_token_b64", op="shared", B=64, groups=1, N=1, full=True, Hq=32, Hkv=8,
             d=128, block=64, pre_lo=4352, pre_hi=4352, own_lo=100, own_hi=1000, lens=7),
        # eight prompts, four images each, two rows of a 24x24 grid as drafts
        dict(name="shared_drafts_8x4", op="shared", B=32, groups=8, N=48, full=False, Hq=16,
             Hkv=16, d=128, block=32, pre_lo=1500, pre_hi=8000, own_lo=24, own_hi=600, lens=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["quant", "matmul", "matmul", "matmul", "norm", "norm", "shared", "shared",
                     "shared"])
    if op == "quant":
        return dict(op=op, rows=_log_int(rng, 1, 17408), K=_log_int(rng, 64, 16384),
                    block_rows=rng.choice([1, 1, 1, 128]), bf16=rng.random() < 0.7,
                    gap=rng.choice([0, 0, 8, 40]))
    if op == "matmul":
        M = rng.choice([_log_int(rng, 1, 128), _log_int(rng, 1, 2048), _log_int(rng, 64, 17408)])
        return dict(op=op, M=M, N=_log_int(rng, 64, 65536), K=_log_int(rng, 64, 12288),
                    bf16=rng.random() < 0.7, add=rng.random() < 0.3, gap=rng.choice([0, 0, 16, 80]))
    heads = [(8, 8, 64), (16, 16, 128), (32, 8, 128), (32, 32, 128), (12, 4, 64), (6, 2, 128)]
    Hq, Hkv, d = rng.choice(heads)
    block = rng.choice([16, 32, 64, 64, 128])
    if op == "norm":
        W = rng.choice([16, 24, 32, 48, 64, rng.randrange(16, 65)])
        prefix = rng.randrange(16, 257)
        full = prefix + W * W
        N = min(rng.choice([1, _log_int(rng, 1, 128), _log_int(rng, 64, 1088)]), full)
        c = dict(op=op, H=W, W=W, prefix=prefix, B=_log_int(rng, 1, 32), N=N, Hq=Hq, Hkv=Hkv, d=d,
                 block=block, len_hi=rng.randrange(0, full - N + 1), lens=rng.randrange(1 << 20),
                 interleaved=rng.random() < 0.5, layer=rng.random() < 0.5,
                 per_head=rng.random() < 0.5)
        c["len_lo"] = rng.randrange(0, c["len_hi"] + 1)
        return c
    groups = _log_int(rng, 1, 16)
    c = dict(op=op, B=groups * _log_int(rng, 1, 64), groups=groups,
             N=rng.choice([1, 1, _log_int(rng, 1, 64)]), full=rng.random() < 0.6, Hq=Hq, Hkv=Hkv,
             d=d, block=block, pre_hi=_log_int(rng, 64, 32768), own_hi=_log_int(rng, 8, 4096),
             lens=rng.randrange(1 << 20))
    c["pre_lo"] = rng.choice([0, c["pre_hi"] // 2, c["pre_hi"]])
    c["own_lo"] = rng.randrange(0, c["own_hi"] + 1)
    return c


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op)
            for op in ("quant", "matmul", "norm", "shared")}
    while True:
        c = _draw(rng)
        if c["op"] == "shared" and _gathered(c) > 3e9:  # (what the plain form lays out)
            continue
        if _cost(c) <= most[c["op"]]:
            return c


def _lengths(case):
    """Cache length and new tokens of every sequence of a "norm" case."""
    r = random.Random(case["lens"])
    B, N = case["B"], case["N"]
    cache = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(B)]
    new = [N if r.random() < 0.25 else r.randint((N + 7) // 8, N) for _ in range(B)]
    if B > 2:
        new[r.randrange(B)] = 0  # a sequence that has nothing new
    return cache, new


def _members(case):
    """Of a "shared" case: the groups' first sequences (and B), shared blocks of every group,
    cache length and new tokens of every sequence."""
    r = random.Random(case["lens"])
    B, n, S, N = case["B"], case["groups"], case["block"], case["N"]
    if case["full"]:
        start = [B * i // n for i in range(n)] + [B]
    else:  # groups of unequal size
        start = [0] + sorted(r.sample(range(1, B), n - 1)) + [B]
    shared = [r.randint(case["pre_lo"], case["pre_hi"]) // S for _ in range(n)]
    cache, new = [], []
    for g in range(n):
        for _ in range(start[g], start[g + 1]):
            cache.append(shared[g] * S + r.randint(case["own_lo"], case["own_hi"]))
            new.append(N if case["full"] or r.random() < 0.5 else r.randint((N + 7) // 8, N))
    if B > 4 and not case["full"]:
        new[r.randrange(B)] = 0  # a sequence that is done
    return start, shared, cache, new


def _blocks(n, block):
    return -(-n // block)


def _gathered(case):
    """Floats of the keys as the plain form lays them out."""
    _, _, cache, new = _members(case)
    return case["B"] * case["Hkv"] * case["d"] * max(c + n for c, n in zip(cache, new))


def work(case):
    if case["op"] == "quant":
        rows, K = case["rows"], case["K"]
        return dict(bytes=rows * K * (2 if case["bf16"] else 4) + rows * K
                    + 4 * _blocks(rows, case["block_rows"]) * _blocks(K, G128), flops=2 * rows * K)
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        kb = _blocks(K, G128)
        out = (2 if case["bf16"] else 4) + (2 if case["add"] else 0)
        return dict(bytes=M * K + N * K + 4 * kb * (M + _blocks(N, G128)) + M * N * out,
                    flops=2 * M * N * K)
    Hq, Hkv, d, S = case["Hq"], case["Hkv"], case["d"], case["block"]
    if case["op"] == "norm":
        cache, new = _lengths(case)
        T = sum(new)
        touched = sum(_blocks(c + n, S) - c // S for c, n in zip(cache, new) if n)
        return dict(bytes=T * (Hq + 2 * Hkv) * d * 2 + 20 * T + T * Hq * d * 2 + T * 2 * Hkv * d
                    + touched * Hkv * 8, flops=8 * T * (Hq + Hkv) * d + 4 * T * Hkv * d)
    start, shared, cache, new = _members(case)
    T = sum(new)
    keys = sum(shared[g] * S for g in range(case["groups"]) if sum(new[start[g]:start[g + 1]]))
    for g in range(case["groups"]):
        keys += sum(cache[b] + new[b] - shared[g] * S for b in range(start[g], start[g + 1]) if new[b])
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(cache, new))
    return dict(bytes=keys * Hkv * 2 * d + 8 * Hkv * (keys // S) + 2 * T * Hq * d * 2,
                flops=4 * d * Hq * pairs)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 300)


# ---------------------------------------------------------------------- prepare
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _values(gen, shape, dtype):
    """Projections as layers give them: normal, heads of unequal size, a few wide channels."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x *= torch.exp(0.3 * torch.randn((shape[-2], 1), generator=gen, device=DEV))
    wide = torch.rand(shape[-1], generator=gen, device=DEV) < 0.03
    return (x * torch.where(wide, 3.0, 1.0)).to(dtype)


def _strided(x, ld):
    """x [rows, n] as the first columns of a wider buffer."""
    if ld == x.shape[1]:
        return x
    y = torch.zeros((x.shape[0], ld), dtype=x.dtype, device=DEV)
    y[:, :x.shape[1]] = x
    return y


def _fill(gen, pool, Hkv, S, d):
    """A cache that earlier tokens filled: values within their scales."""
    scale = 0.004 * torch.exp(0.3 * torch.randn((pool, Hkv), generator=gen, device=DEV))
    x = torch.randn((pool, Hkv, S, d), generator=gen, device=DEV)
    return (x / scale[:, :, None, None]).clamp(-TOP, TOP).to(E4M3), scale.contiguous()


def _eighths(x, block_rows):
    """x [rows, K] float32 as e4m3 and the scales [K / 128, rows / block_rows]."""
    rows, K = x.shape
    R, C = _blocks(rows, block_rows), _blocks(K, G128)
    y = torch.zeros((R * block_rows, C * G128), device=DEV)
    y[:rows, :K] = x
    y = y.view(R, block_rows, C, G128)
    scale = y.abs().amax((1, 3)).clamp(min=FLOOR) / TOP
    q = (y * (1.0 / scale)[:, None, :, None]).clamp(-TOP, TOP)
    return q.view(R * block_rows, C * G128)[:rows, :K].to(E4M3), scale.t().contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1000003 + 29)
    s = dict(case=dict(case), status=torch.zeros(1, dtype=torch.int32, device=DEV))
    return globals()["prepare_" + case["op"]](s, case, gen)


def prepare_quant(s, case, gen):
    rows, K = case["rows"], case["K"]
    x = _values(gen, (rows, K), torch.bfloat16 if case["bf16"] else torch.float32)
    s["ldx"], s["ldo"] = (K + 7) // 8 * 8 + case["gap"], (K + 15) // 16 * 16
    s["x"] = _strided(x, s["ldx"])
    s["out"] = torch.zeros((rows, s["ldo"]), dtype=E4M3, device=DEV)
    s["scale"] = torch.zeros((_blocks(K, G128), _blocks(rows, case["block_rows"])), device=DEV)
    return s


def prepare_matmul(s, case, gen):
    M, N, K = case["M"], case["N"], case["K"]
    ld = (K + 15) // 16 * 16
    s["lda"], s["ldw"], s["ldc"] = ld + case["gap"], ld, N + case["gap"]
    a, s["a_scale"] = _eighths(_values(gen, (M, K), torch.float32), 1)
    w = torch.randn((N, K), generator=gen, device=DEV) * K ** -0.5
    w *= torch.exp(0.3 * torch.randn((N, 1), generator=gen, device=DEV))
    w, s["w_scale"] = _eighths(w, G128)
    s["a"], s["w"] = _strided(a, s["lda"]), _strided(w, s["ldw"])
    s["add"] = torch.randn((M, N), generator=gen, device=DEV).to(torch.bfloat16) if case["add"] else None
    s["c"] = torch.zeros((M, s["ldc"]), dtype=torch.bfloat16 if case["bf16"] else torch.float32,
                         device=DEV)
    return s


def _table(case, gen, rows):
    """Block tables over a pool in random order; rows: lists of numbers that name the blocks."""
    pool = 1 + max([max(r) for r in rows if r], default=0) + 3
    ids = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
    M = max(max(len(r) for r in rows), 1)
    at = _i32([r + [-1] * (M - len(r)) for r in rows])
    return torch.where(at >= 0, ids[at.clamp(min=0).long()], -1).to(torch.int32).contiguous(), pool


def prepare_norm(s, case, gen):
    cache, new = _lengths(case)
    B, N, S = case["B"], case["N"], case["block"]
    Hq, Hkv, d, P, W = case["Hq"], case["Hkv"], case["d"], case["prefix"], case["W"]
    names, n = [], 0
    for c, k in zip(cache, new):
        names.append(list(range(n, n + _blocks(c + k, S))))
        n += len(names[-1])
    table, pool = _table(case, gen, names)
    s["n_new"] = _i32(new)
    s["k"], s["k_scale"] = _fill(gen, pool, Hkv, S, d)
    s["v"], s["v_scale"] = _fill(gen, pool, Hkv, S, d)
    p = _i32(cache).long()[:, None] + torch.arange(N, device=DEV)[None]
    blk = torch.gather(table.long(), 1, (p // S).clamp(max=table.shape[1] - 1))
    live = torch.arange(N, device=DEV)[None] < s["n_new"][:, None]
    s["slots"] = torch.where(live, blk * S + p % S, -1).contiguous()
    i = (p - P).clamp(min=0)
    s["pos"] = torch.stack([torch.where(p < P, p, P), torch.where(p < P, p, P + i // W),
                            torch.where(p < P, p, P + i % W)], -1).to(torch.int32).contiguous()
    # rotary table: a quarter of the pairs by time, the rest by row and column
    pairs = d // 2
    s["sections"] = (pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8)
    freq = 10000.0 ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / pairs)
    angle = torch.arange(P + case["H"] * W + 1, device=DEV,
                         dtype=torch.float64)[:, None] * freq.float().double()[None]
    s["rotary"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
    qkv = _values(gen, (B, N, Hq + 2 * Hkv, d), torch.bfloat16)  # one projection's output
    s["new_q"], s["new_k"], s["new_v"] = qkv.split([Hq, Hkv, Hkv], 2)
    for x, heads in (("q", Hq), ("k", Hkv)):
        shape = (heads, d) if case["per_head"] else (d,)
        s[x + "_gain"] = 1.0 + 0.2 * torch.randn(shape, generator=gen, device=DEV)
        s[x + "_bias"] = 0.1 * torch.randn(shape, generator=gen, device=DEV) if case["layer"] else None
    s["q_out"] = torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device=DEV)
    return s


def prepare_shared(s, case, gen):
    start, shared, cache, new = _members(case)
    B, N, S = case["B"], case["N"], case["block"]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    names, n = [], 0
    for g in range(case["groups"]):
        first = list(range(n, n + shared[g]))
        n += shared[g]
        for b in range(start[g], start[g + 1]):
            more = _blocks(cache[b] + new[b], S) - shared[g]
            names.append(first + list(range(n, n + more)))
            n += more
    s["table"], pool = _table(case, gen, names)
    s["group_start"], s["shared"], s["max_shared"] = _i32(start), _i32(shared), max(shared)
    s["cache_len"], s["n_new"] = _i32(cache), _i32(new)
    s["k"], s["k_scale"] = _fill(gen, pool, Hkv, S, d)
    s["v"], s["v_scale"] = _fill(gen, pool, Hkv, S, d)
    s["q"] = (1.5 * _values(gen, (B, N, Hq, d), torch.float32)).to(torch.bfloat16)
    s["o"] = torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device=DEV)
    return s


# -------------------------------------------------------------------------- run
def run(s):
    return globals()[("own_" if own else "plain_") + s["case"]["op"]](s)


def own_quant(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    ssd.ssd_quantize(c["rows"], c["K"], c["block_rows"], s["x"], s["ldx"], s["out"], s["ldo"],
                     s["scale"], s["scale"].shape[1])
    return dict(out=s["out"][:, :c["K"]], scale=s["scale"])


def plain_quant(s):
    c = s["case"]
    q, scale = _eighths(s["x"][:, :c["K"]].float(), c["block_rows"])
    return dict(out=q, scale=scale)


def own_matmul(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    ssd.ssd_scaled_matmul(c["M"], c["N"], c["K"], s["a"], s["lda"], s["a_scale"], c["M"], s["w"],
                          s["ldw"], s["w_scale"], s["w_scale"].shape[1], s["add"], c["N"], s["c"],
                          s["ldc"], s["status"])
    return dict(c=s["c"][:, :c["N"]], status=s["status"])


def plain_matmul(s):
    c = s["case"]
    M, N, K = c["M"], c["N"], c["K"]
    a = s["a"][:, :K].float() * s["a_scale"].t().repeat_interleave(G128, 1)[:, :K]
    w = s["w"][:, :K].float()
    w *= s["w_scale"].t().repeat_interleave(G128, 1)[:, :K].repeat_interleave(G128, 0)[:N]
    y = torch.matmul(a, w.t())
    if s["add"] is not None:
        y += s["add"].float()
    return dict(c=y.to(s["c"].dtype), status=s["status"])


def own_norm(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    if "cache" not in s:
        s["cache"] = ssd.cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["rot"] = ssd.rotary(s["rotary"], s["sections"], c["interleaved"])
        s["norm"] = ssd.head_norm("layer" if c["layer"] else "rms", 1e-6, s["q_gain"], s["q_bias"],
                                  s["k_gain"], s["k_bias"])
    ssd.ssd_cache_append_norm(s["cache"], s["rot"], s["norm"], c["B"], c["N"], c["Hq"], s["n_new"],
                              s["slots"], s["pos"], s["new_q"], s["new_q"].stride(1), s["new_k"],
                              s["new_k"].stride(1), s["new_v"], s["new_v"].stride(1), s["q_out"],
                              s["status"])
    return dict(q=s["q_out"], k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                status=s["status"])


def _normed(s, x, gain, bias):
    x = x.float()
    if s["case"]["layer"]:
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain
    return x if bias is None else x + bias


def _rotate(s, x):
    c = s["case"]
    sec = s["sections"]
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(sec, device=DEV))
    rows = s["pos"].long()[:, :, axis]
    cs = s["rotary"][rows, torch.arange(sum(sec), device=DEV)]
    cos, sin = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
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
    grown = touched & (~kept | (m > TOP * scale))
    new_scale = torch.where(grown, m.clamp(min=FLOOR) / TOP, scale)
    inv = 1.0 / new_scale
    factor = (scale * inv)[:, :, None, None]
    again = (kept & grown)[:, :, None, None] & (torch.arange(S, device=DEV)[:, None]
                                                < first[:, :, None, None])
    cache = torch.where(again, (cache.float() * factor).to(E4M3).float(), cache.float())
    cache[blk, :, off] = (x * inv[blk][:, :, None]).clamp(-TOP, TOP).to(E4M3).float()
    return cache.to(E4M3), new_scale


def plain_norm(s):
    q = _rotate(s, _normed(s, s["new_q"], s["q_gain"], s["q_bias"])).to(torch.bfloat16)
    q = torch.where((s["slots"] >= 0)[:, :, None, None], q, 0)
    k, ks = _write(s, _rotate(s, _normed(s, s["new_k"], s["k_gain"], s["k_bias"])), s["k"],
                   s["k_scale"])
    v, vs = _write(s, s["new_v"].float(), s["v"], s["v_scale"])
    return dict(q=q, k=k, v=v, k_scale=ks, v_scale=vs, status=s["status"])


def own_shared(s):
    import paper_2606_20543_gb300 as ssd
    c = s["case"]
    M = s["table"].shape[1]
    if "grid" not in s:
        s["grid"] = ssd.grid(64, 64, 0)
        s["cache"] = ssd.cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        n = ssd.ssd_cache_attention_shared_workspace(c["B"], c["groups"], c["Hq"], c["Hkv"], c["d"],
                                                     c["N"], M * c["block"],
                                                     s["max_shared"] * c["block"])
        s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device=DEV)
    ssd.ssd_cache_attention_shared(s["grid"], s["cache"], c["B"], c["groups"], s["group_start"],
                                   s["shared"], s["max_shared"], c["Hq"], s["cache_len"], s["n_new"],
                                   None, None, c["N"], s["table"], M, s["q"], 0.0, s["o"], None,
                                   s["ws"], s["ws"].numel(), s["status"])
    return dict(o=s["o"], status=s["status"])


def plain_shared(s):
    c = s["case"]
    B, N, Hq, Hkv, d, S = c["B"], c["N"], c["Hq"], c["Hkv"], c["d"], c["block"]
    L, G = s["table"].shape[1] * S, Hq // Hkv

    def gathered(x, scale):
        at = s["table"].long().clamp(min=0)
        y = x[at].float()                                            # [B, M, Hkv, S, d]
        y *= scale[at][:, :, :, None, None]
        return y.transpose(1, 2).reshape(B, Hkv, L, d)

    at = torch.arange(L, device=DEV)[None]
    end = s["cache_len"] + s["n_new"]
    k = gathered(s["k"], s["k_scale"])
    k.masked_fill_((at >= end[:, None])[:, None, :, None], 0.0)
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
    v = gathered(s["v"], s["v_scale"])
    v.masked_fill_((at >= end[:, None])[:, None, :, None], 0.0)
    o = torch.matmul(x, v).reshape(B, Hkv, N, G, d).permute(0, 2, 1, 3, 4)
    return dict(o=o.reshape(B, N, Hq, d).to(torch.bfloat16), status=s["status"])


# ------------------------------------------------------------------------ exact
def exact(case, seed):
    s = prepare(case, seed)
    return globals()["exact_" + case["op"]](s)


def _round8(x):
    """The nearest e4m3 value, ties to even, in 64 bits."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6.0)
    step = torch.exp2(e - 3.0)
    return (torch.round(x / step) * step).clamp(-TOP, TOP)


def exact_quant(s):
    """A column of blocks after the other."""
    c = s["case"]
    rows, K, R = c["rows"], c["K"], c["block_rows"]
    out = torch.zeros((rows, K), dtype=torch.float64, device=DEV)
    scale = torch.zeros(s["scale"].shape, dtype=torch.float64, device=DEV)
    which = torch.arange(rows, device=DEV) // R
    for i in range(scale.shape[0]):
        x = s["x"][:, i * G128:min(K, (i + 1) * G128)].double()
        m = torch.zeros(scale.shape[1], dtype=torch.float64, device=DEV)
        m.scatter_reduce_(0, which, x.abs().amax(1), "amax")
        scale[i] = m.clamp(min=FLOOR) / TOP
        out[:, i * G128:min(K, (i + 1) * G128)] = _round8(x / scale[i][which][:, None])
    return dict(out=out, scale=scale)


def exact_matmul(s):
    """A block of 128 of the inner length after the other."""
    c = s["case"]
    M, N, K = c["M"], c["N"], c["K"]
    if M * N * K > 2e12:
        return None
    y = torch.zeros((M, N), dtype=torch.float64, device=DEV)
    col = torch.arange(N, device=DEV) // G128
    for i in range(_blocks(K, G128)):
        at = slice(i * G128, min(K, (i + 1) * G128))
        a = s["a"][:, at].double() * s["a_scale"][i].double()[:, None]
        w = s["w"][:, at].double() * s["w_scale"][i].double()[col][:, None]
        y.addmm_(a, w.t())
    if s["add"] is not None:
        y += s["add"].double()
    return dict(c=y, status=None)


def exact_norm(s):
    """Head norms by their definition, positions as complex factors, the cache block by block."""
    c = s["case"]
    S, d, Hkv = c["block"], c["d"], c["Hkv"]
    cache_len, new = _lengths(c)
    sec, pairs = s["sections"], d // 2
    axis = [0] * sec[0] + [1] * sec[1] + [2] * sec[2]
    freq = torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], dtype=torch.float64,
                        device=DEV).float().double()
    t = s["pos"][:, :, axis].double() * freq
    z = torch.polar(torch.ones_like(t), t)[:, :, None]

    def turned(x, gain, bias):
        x = x.double()
        if c["layer"]:
            var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            x = (x - mean) / torch.sqrt(var + 1e-6)
        else:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + 1e-6)
        x = x * gain.double() + (0.0 if bias is None else bias.double())
        a, b = (x[..., 0::2], x[..., 1::2]) if c["interleaved"] else (x[..., :pairs], x[..., pairs:])
        y = torch.complex(a, b) * z
        return (torch.stack([y.real, y.imag], -1).flatten(-2) if c["interleaved"]
                else torch.cat([y.real, y.imag], -1))

    q = turned(s["new_q"], s["q_gain"], s["q_bias"])
    out = dict(q=q, status=None)
    for name, x in (("k", turned(s["new_k"], s["k_gain"], s["k_bias"])), ("v", s["new_v"].double())):
        cache, scale = s[name].double(), s[name + "_scale"].double()
        for b, (at, n) in enumerate(zip(cache_len, new)):
            q[b, n:] = 0
            for i in range(at // S, _blocks(at + n, S) if n else 0):
                lo, hi = max(at, i * S), min(at + n, (i + 1) * S)
                blk = int(s["slots"][b, lo - at]) // S
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


def exact_shared(s):
    c = s["case"]
    G, d = c["Hq"] // c["Hkv"], c["d"]
    _, _, cache, new = _members(c)
    if c["B"] * c["Hkv"] > 2048:
        return None
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV)
    for b, (at, n) in enumerate(zip(cache, new)):
        blocks = s["table"][b, :_blocks(at + n, c["block"])].long()
        for g in range(c["Hkv"] if n else 0):
            k, v = ((s[x][blocks, g].double() * s[x + "_scale"][blocks, g].double()[:, None, None])
                    .reshape(-1, d)[:at + n] for x in ("k", "v"))
            x = torch.einsum("nhd,sd->nhs", s["q"][b, :n, g * G:(g + 1) * G].double(), k)
            hide = torch.ones((n, at + n), dtype=torch.bool, device=DEV).triu(at + 1)
            p = torch.softmax((x / math.sqrt(d)).masked_fill(hide[:, None], -math.inf), -1)
            o[b, :n, g * G:(g + 1) * G] = torch.einsum("nhs,sd->nhd", p, v)
    return dict(o=o, status=None)
