"""ssd_scaled_matmul on all finite e4m3 codes, up to 448 (every quantised block holds its largest there),
with the scales that ssd_quantize gives blocks of zeros; and calls of every kernel on two streams at
once.  Tolerance as in tests/test_gpu_scaled_matmul.py: (132 + blocks) 2^-23 of the sum of the terms'
magnitudes, and half a step of the result."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import scaled as oq
from tests.test_gpu_scaled_matmul import Case, up

pytestmark = pytest.mark.gpu

ZERO = np.float32(oc.LEAST / oc.TOP)  # the scale of a block of zeros


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


def finite(rng, shape):
    x = rng.integers(0, 256, shape).astype(np.uint8)
    x[(x & 0x7f) == 0x7f] ^= 1  # (448 in the place of NaN)
    return x


@pytest.mark.parametrize("M,N,K", [(3, 100, 2048), (16, 20011, 300), (24, 1000, 2100), (40, 300, 300),
                                   (60, 700, 4200), (200, 1000, 2100), (1500, 2049, 700), (2100, 2304, 2100)])
@pytest.mark.parametrize("kind", ["all", "top", "zeros"])
def test_all_finite_codes(ssd, M, N, K, kind):
    c, rng = Case(M, N, K, 41), np.random.default_rng(M + N)
    a, w = finite(rng, (M, K)), finite(rng, (N, K))
    if kind == "top":  # some blocks of +-448 alone
        for x in (a, w):
            x[::3, :128] = np.where(x[::3, :128] & 0x80, 0xfe, 0x7e)
    if kind == "zeros":  # rows of A, and blocks of W, of zeros of either sign
        a[::2] &= 0x80
        w[128:256, :128] &= 0x80
        c.sa[:, :M:2], c.sw[0, 1:2] = ZERO, ZERO
    c.a[:, :K], c.w[:, :K] = a, w
    for n in ("a", "w", "sa", "sw"):
        c.dev[n] = torch.from_numpy(getattr(c, n)).cuda()
    assert (oc.TABLE[a].max() == 448) and (oc.TABLE[w].max() == 448)
    c.check(ssd, True)
    c.check(ssd, False, add=True)


def test_products_of_every_kernel_at_once(ssd):
    """On two streams, every call into a buffer of its own: what each gives alone."""
    sizes = [(5, 1500, 2100), (16, 30000, 700),      # 16 columns, cut over a cluster and not
             (24, 1000, 2100), (24, 40000, 300),     # 32
             (40, 3000, 2100), (50, 40000, 260),     # 64
             (200, 1000, 2100), (2100, 2304, 2100),  # 128 x 128, 256 x 128 of a pair,
             (2304, 4096, 1000), (1500, 2049, 2100)]  # 256 x 256, and with rows of C anywhere
    cases = [Case(M, N, K, 7 * M) for M, N, K in sizes]
    rounds, streams = 6, [torch.cuda.Stream() for _ in range(2)]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(c, out, stream=None):
        ssd.ssd_scaled_matmul(c.M, c.N, c.K, c.dev["a"], c.lda, c.dev["sa"], c.ldas, c.dev["w"], c.ldw,
                              c.dev["sw"], c.ldws, None, 0, out, c.N, st, stream=stream)

    alone, out = [], []
    for c in cases:
        o = torch.full((c.M, c.N), 7.0, dtype=torch.bfloat16, device="cuda")
        call(c, o)
        torch.cuda.synchronize()
        alone.append(o)
        out.append(torch.full((rounds,) + o.shape, 7.0, dtype=o.dtype, device="cuda"))
        a, w = oc.TABLE[c.a[:3, :c.K]], oc.TABLE[c.w[:, :c.K]]
        want, mag = oq.matmul(a, c.sa[:, :3].astype(np.float64), w, c.sw.astype(np.float64)[:, :up(c.N, 128) // 128])
        assert (np.abs(o[:3].double().cpu().numpy() - want)
                <= (132 + len(c.sa)) * 2.0 ** -23 * mag + 2.0 ** -8 * np.abs(want)).all()
    torch.cuda.synchronize()
    for r in range(rounds):
        for i in range(len(cases)):
            j = (i + r) % len(cases)
            call(cases[j], out[j][r], streams[i % 2])
    torch.cuda.synchronize()
    assert st.item() == 0
    for o, a in zip(out, alone):
        for x in o:
            assert torch.equal(x.view(torch.int16), a.view(torch.int16))
