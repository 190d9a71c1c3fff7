"""ssd_quantize against its float64 definition (oracle/scaled.py).

Tolerances: a scale is a float32 quotient of a value that is one already: 2^-24 of it.  1 / s and
the product with it round twice more, so an entry is a neighbour of its unrounded value: half the
e4m3 step, and 2^-22 of the value for three roundings of 2^-24."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import scaled as oq

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


def up(x, n):
    return -(-x // n) * n


def quantized(ssd, x, block_rows, gap=0):
    """x [rows, K] on the GPU: codes uint8 [rows, ldo], scales [C, lds], with what lies beside."""
    rows, K = x.shape
    ldx, ldo = up(K, 8) + gap, up(K, 16) + 2 * gap
    C, R = up(K, 128) // 128, up(rows, block_rows) // block_rows
    buf = torch.full((rows, ldx), float("nan"), dtype=x.dtype, device="cuda")
    buf[:, :K] = x
    flat = buf.flatten()[:(rows - 1) * ldx + K].clone()  # (ends with the last value)
    out = torch.full((rows, ldo), 0x5a, dtype=torch.uint8, device="cuda")
    scale = torch.full((C, R + gap), -3.0, device="cuda")
    ssd.ssd_quantize(rows, K, block_rows, flat, ldx, out, ldo, scale, R + gap)
    torch.cuda.synchronize()
    return out.cpu().numpy(), scale.cpu().numpy()


def check(ssd, x, block_rows, gap=0):
    rows, K = x.shape
    out, scale = quantized(ssd, x.cuda(), block_rows, gap)
    want, s = oq.quantize(x.double().numpy(), block_rows)
    R = s.shape[1]
    assert (np.abs(scale[:, :R] - s) <= 2.0 ** -24 * s).all()
    assert (scale[:, R:] == -3.0).all() and (out[:, K:] == 0x5a).all()
    got = oc.TABLE[out[:, :K]]
    nan = np.isnan(want)
    assert np.array_equal(nan, np.isnan(got))
    tol = 0.5 * oc.e4m3_step(want) + 2.0 ** -22 * np.abs(want)
    assert (np.abs(got - want) <= tol)[~nan].all()


@pytest.mark.parametrize("rows,K", [(1, 1), (1, 128), (3, 129), (8, 4096), (33, 2050), (127, 513),
                                    (128, 16), (129, 1000), (300, 64), (1000, 143)])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sizes(ssd, rows, K, block_rows, dtype):
    g = torch.Generator().manual_seed(rows * K)
    x = torch.randn((rows, K), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))
    check(ssd, x.to(dtype), block_rows, gap=0 if K % 2 else 40)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_zeros_nan_infinities_and_extremes(ssd, block_rows, dtype):
    g = torch.Generator().manual_seed(3)
    x = torch.randn((130, 300), generator=g).to(dtype)
    x[0] = 0.0
    x[1, 5], x[1, 6], x[1, 7] = float("nan"), float("inf"), -float("inf")
    x[2] = float("nan")
    x[3] = float("inf")
    x[4, :128], x[4, 128:] = 1e-38, -3e38
    x[129] *= 2.0 ** -90
    check(ssd, x, block_rows)


def test_every_e4m3_value_stays(ssd):
    """Entries that are e4m3 values beside a largest of 448 come back as they were."""
    codes = np.array([c for c in range(256) if (c & 0x7f) != 0x7f], np.uint8)
    x = torch.from_numpy(oc.TABLE[codes].astype(np.float32))[None].contiguous()
    out, scale = quantized(ssd, torch.cat([x, x, x, x[:, :2]], 1).cuda()[:, :640], 1)
    x4 = np.concatenate([codes, codes, codes])[:640]
    whole = np.isclose(scale[:, 0], 1.0, rtol=0, atol=0)
    for j in np.nonzero(whole)[0]:
        assert np.array_equal(out[0, j * 128:(j + 1) * 128], x4[j * 128:(j + 1) * 128])
    assert whole.sum() >= 2


def test_offsets_beyond_32_bits(ssd):
    """More than 2^31 entries: the last rows as rows of a small call."""
    rows, K = 300000, 8192
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    x[-200:].normal_()
    for block_rows in (1, 128):
        R = -(-rows // block_rows)
        out = torch.zeros((rows, K), dtype=torch.uint8, device="cuda")
        scale = torch.zeros((K // 128, R), device="cuda")
        ssd.ssd_quantize(rows, K, block_rows, x, K, out, K, scale, R)
        at = rows // 128 * 128 - 128
        part, few = torch.zeros((rows - at, K), dtype=torch.uint8, device="cuda"), -(-(rows - at) // block_rows)
        want = torch.zeros((K // 128, few), device="cuda")
        ssd.ssd_quantize(rows - at, K, block_rows, x[at:], K, part, K, want, few)
        torch.cuda.synchronize()
        assert torch.equal(out[at:], part) and torch.equal(scale[:, -few:], want)
        assert (part[-100:] != 0).any()
        del out


def test_graph_and_stream(ssd):
    x = torch.randn((64, 512), device="cuda")
    out, scale = torch.zeros((64, 512), dtype=torch.uint8, device="cuda"), torch.zeros((4, 64), device="cuda")
    ssd.ssd_quantize(64, 512, 1, x, 512, out, 512, scale, 64)
    torch.cuda.synchronize()
    want = out.clone(), scale.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ssd.ssd_quantize(64, 512, 1, x, 512, out, 512, scale, 64)
    x.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(scale, 2 * want[1])
