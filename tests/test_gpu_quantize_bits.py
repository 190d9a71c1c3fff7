"""ssd_quantize bit for bit: its formula (include/ssd.h) in float32, every step rounded once, as numpy
computes it.  (Against 64 bits entries next to a border between two e4m3 values go either way, as they
do in any float32 evaluation.)"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


def formula(x, block_rows):
    """x float32 [rows, K]: codes [rows, K] and scales [ceil(K / 128), ceil(rows / block_rows)]."""
    rows, K = x.shape
    codes = np.zeros((rows, K), np.uint8)
    scale = np.zeros((-(-K // 128), -(-rows // block_rows)), np.float32)
    for i in range(scale.shape[1]):
        for j in range(scale.shape[0]):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]
            m = np.abs(x[at]).max()
            s = np.float32(max(m, np.float32(2.0 ** -100)) / np.float32(448))
            y = np.clip(x[at] * (np.float32(1) / s), np.float32(-448), np.float32(448))
            codes[at] = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            scale[j, i] = s
    return codes, scale


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,K", [(1, 128), (300, 1000), (129, 4096)])
def test_bits(ssd, rows, K, block_rows, bf16):
    rng = np.random.default_rng(rows + K)
    x = (rng.standard_normal((rows, K)) * np.exp(3 * rng.standard_normal((rows, 1)))).astype(np.float32)
    x = torch.from_numpy(x).to(torch.bfloat16 if bf16 else torch.float32)
    want, scales = formula(x.float().numpy(), block_rows)
    ldo = -(-K // 16) * 16
    out = torch.zeros((rows, ldo), dtype=torch.uint8, device="cuda")
    scale = torch.zeros(scales.shape, device="cuda")
    ssd.ssd_quantize(rows, K, block_rows, x.cuda(), K, out, ldo, scale, scale.shape[1])
    torch.cuda.synchronize()
    assert np.array_equal(scale.cpu().numpy().view(np.uint32), scales.view(np.uint32))
    assert np.array_equal(out.cpu().numpy()[:, :K], want)
