"""Linear layers whose inputs and weights are e4m3 with a float32 scale per 128 entries: a weight
laid out once, inputs quantised at the call.

Marshalling only, on torch's current stream; nothing waits for the device, so calls can be captured
in a CUDA graph.  What went wrong on the device is in ``status`` (include/ssd.h)."""
from __future__ import annotations

import torch

from . import ssd_quantize, ssd_scaled_matmul

GROUP = 128


def _up(x, n):
    return -(-x // n) * n


class ScaledRows:
    """Up to ``rows`` rows of ``K`` values as e4m3 with a scale per 128 (a buffer to quantise into).
    Rows that several layers read are quantised once."""

    def __init__(self, rows, K, device="cuda"):
        self.rows, self.K, self.ld = rows, K, _up(K, 16)
        self.q = torch.zeros((rows, self.ld), dtype=torch.float8_e4m3fn, device=device)
        self.scale = torch.zeros((-(-K // GROUP), rows), dtype=torch.float32, device=device)
        self.M = 0

    def quantize(self, x):
        """x bf16 or float32 [M, K], M at most rows; rows may lie apart (a multiple of 8 values, the
        first 16-byte aligned).  Returns self."""
        M, K = x.shape
        if K != self.K or M > self.rows or (K > 1 and x.stride(1) != 1):
            raise ValueError("x: at most %d rows of %d values side by side" % (self.rows, self.K))
        ld = x.stride(0) if M > 1 else _up(K, 8)
        ssd_quantize(M, K, 1, x, ld, self.q, self.ld, self.scale, self.rows)
        self.M = M
        return self


class ScaledLinear:
    """y = x W^T (+ add) of a weight [N, K] (bf16 or float32), which is quantised here, with a scale
    for every block of 128 x 128."""

    def __init__(self, weight, status=None):
        N, K = weight.shape
        if weight.stride(1) != 1 or weight.stride(0) % 8 != 0 or weight.stride(0) < K or weight.data_ptr() % 16:
            weight = torch.cat([weight, weight.new_zeros((N, -K % 8))], 1)  # (a copy in any case)
        self.N, self.K, self.ld = N, K, _up(K, 16)
        dev = weight.device
        self.w = torch.zeros((N, self.ld), dtype=torch.float8_e4m3fn, device=dev)
        self.scale = torch.zeros((-(-K // GROUP), -(-N // GROUP)), dtype=torch.float32, device=dev)
        ssd_quantize(N, K, GROUP, weight, weight.stride(0), self.w, self.ld, self.scale, self.scale.shape[1])
        self.status = torch.zeros((1,), dtype=torch.int32, device=dev) if status is None else status

    def __call__(self, x: ScaledRows, add=None, out=None, dtype=torch.bfloat16):
        """x quantised rows; add bf16 [M, N] or None; out [M, N] bf16 or float32 (a new tensor of
        ``dtype`` if None; may be ``add``).  Rows of add and out may lie apart."""
        M, N = x.M, self.N
        if x.K != self.K:
            raise ValueError("x has %d columns, the weight %d" % (x.K, self.K))
        if out is None:
            out = torch.empty((M, N), dtype=dtype, device=self.w.device)
        for t in (out, add):
            if t is not None and (tuple(t.shape) != (M, N) or (N > 1 and t.stride(1) != 1)):
                raise ValueError("add and out: [M, N], entries side by side")
        ld = lambda t: N if t is None or M < 2 else t.stride(0)  # noqa: E731
        ssd_scaled_matmul(M, N, self.K, x.q, x.ld, x.scale, x.rows, self.w, self.ld, self.scale,
                          self.scale.shape[1], add, ld(add), out, ld(out), self.status)
        return out
