"""Images decoded token by token over the paged 8-bit cache, on random weights:
the prompts in one pass, then one CUDA graph per token (plan, per layer append
and attention, sampling).

    python examples/paged_decode.py --batch 8 --grid 32 --prefix 64
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2606_20543_gb300 as ssd  # noqa: E402
from paper_2606_20543_gb300.decode import PagedDecode  # noqa: E402


class Toy:
    """A decoder of the usual form with random weights, its products torch's."""

    def __init__(self, V, layers, Hq, Hkv, d, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        width = Hq * d

        def w(*shape):
            x = torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5
            return x.to(torch.bfloat16)

        self.Hq, self.Hkv, self.d = Hq, Hkv, d
        self.embed, self.head = w(V, width) * V ** 0.5, w(width, V)
        self.qkv = [w(width, (Hq + 2 * Hkv) * d) for _ in range(layers)]
        self.out = [w(width, width) for _ in range(layers)]

    def __call__(self, dec: PagedDecode, tokens, last=None):
        """Logits of every row of tokens [B * N], or of the rows `last`."""
        x = self.embed[tokens]
        a, b = self.Hq * self.d, (self.Hq + self.Hkv) * self.d
        for i in range(len(self.qkv)):
            h = x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)
            y = h @ self.qkv[i]
            x = x + dec.attend(i, y[:, :a], y[:, a:b], y[:, b:]) @ self.out[i]
        if last is not None:
            x = x[last]
        h = x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)
        return h @ self.head


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--grid", type=int, default=32)
    p.add_argument("--prefix", type=int, default=64)
    p.add_argument("--vocab", type=int, default=16384)
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--heads", type=int, nargs=3, default=(16, 4, 128), metavar=("HQ", "HKV", "D"))
    p.add_argument("--block", type=int, default=64)
    p.add_argument("--top-k", type=int, default=2000)
    p.add_argument("--top-p", type=float, default=0.95)
    p.add_argument("--seed", type=int, default=1)
    p.add_argument("--no-graph", action="store_true", help="launch every token's kernels one by one")
    a = p.parse_args(argv)
    Hq, Hkv, d = a.heads
    B, total = a.batch, a.prefix + a.grid * a.grid
    per_seq = -(-total // a.block)
    pairs = d // 2
    freq = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().cuda()
    dec = PagedDecode(ssd.grid(a.grid, a.grid, a.prefix), B, Hq, Hkv, d, B * per_seq, a.block,
                      per_seq, a.prefix, freq, (pairs - 2 * (pairs // 3), pairs // 3, pairs // 3),
                      layers=a.layers)
    model = Toy(a.vocab, a.layers, Hq, Hkv, d, a.seed)
    gen = torch.Generator("cuda").manual_seed(a.seed)
    prompt = torch.randint(0, a.vocab, (B * a.prefix,), generator=gen, device="cuda")
    uniforms = torch.rand((a.grid * a.grid, B, 2), generator=gen, device="cuda")
    settings = ssd.sampling(1.0, a.top_k, a.top_p)
    image = torch.empty((a.grid * a.grid, B), dtype=torch.int32, device="cuda")

    # ---- the prompts, and the first token
    u = torch.empty((B, 2), device="cuda")
    rng = ssd.rng(uniforms=u)
    u.copy_(uniforms[0])
    dec.plan(torch.full((B,), a.prefix, dtype=torch.int32, device="cuda"))
    last = torch.arange(1, B + 1, device="cuda") * a.prefix - 1
    tok = dec.sample(model(dec, prompt, last), settings, rng).clone()
    dec.advance()
    image[0] = tok

    # ---- a token of every image
    one = torch.ones((B,), dtype=torch.int32, device="cuda")

    def step():
        dec.plan(one, 1)
        tok.copy_(dec.sample(model(dec, tok), settings, rng))
        dec.advance()

    u.copy_(uniforms[1])
    step()  # (also what a capture needs done before it)
    image[1] = tok
    graph = None
    if not a.no_graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for i in range(2, a.grid * a.grid):
        u.copy_(uniforms[i])
        if graph is None:
            step()
        else:
            graph.replay()
        image[i] = tok
    torch.cuda.synchronize()
    dt = time.perf_counter() - t0
    if int(dec.status.item()) != 0:
        raise RuntimeError("device status %d" % int(dec.status.item()))
    n = a.grid * a.grid - 2
    pool = 2 * dec.k.numel() + 8 * dec.k_scale.numel()
    print("%d images of %d x %d: %.1f us a token, %.0f tokens/s; cache %.1f MB (bf16: %.1f MB)"
          % (B, a.grid, a.grid, dt / n * 1e6, n * B / dt, pool / 1e6, 4 * dec.k.numel() / 1e6))
    dec.release(torch.ones((B,), dtype=torch.bool, device="cuda"))
    return image.t().cpu()


if __name__ == "__main__":
    main()
