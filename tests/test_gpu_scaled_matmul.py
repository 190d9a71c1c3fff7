"""ssd_scaled_matmul against its float64 definition (oracle/scaled.py).

Tolerances: products of e4m3 are exact in float32.  A block's sum makes 127 additions in some order,
each off by at most 2^-23 of the terms' magnitudes (also if it truncates), its scales two roundings,
the sum over the blocks one each, add one: (132 + blocks) 2^-23 of the sum of the terms' magnitudes.
Rounding to bf16 is half a step, 2^-8 of the value, to float32 2^-24."""
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


class Case:
    """Codes and scales on the GPU, in wider buffers whose rest is NaN."""

    def __init__(self, M, N, K, seed=0, gap=16, offset=0, spread=1.0, ldc=None):
        rng = np.random.default_rng(seed)
        self.M, self.N, self.K, C = M, N, K, up(K, 128) // 128

        def codes(rows, ld):
            x = np.full((rows, ld), 0x7f, np.uint8)
            y = rng.integers(0, 256, (rows, K)).astype(np.uint8)
            y[(y & 0x7f) >= 0x70] &= 0xbf  # (nothing above 28, no NaN)
            x[:, :K] = y
            return x

        self.lda, self.ldw = up(K, 16) + gap, up(K, 16) + 2 * gap
        self.a, self.w = codes(M, self.lda), codes(N, self.ldw)
        self.ldas, self.ldws = M + gap, up(N, 128) // 128 + gap
        self.sa = np.exp(spread * rng.standard_normal((C, self.ldas))).astype(np.float32)
        self.sw = np.exp(spread * rng.standard_normal((C, self.ldws))).astype(np.float32)
        self.sa[:, M:], self.sw[:, up(N, 128) // 128:] = np.nan, np.nan
        self.add = torch.from_numpy(rng.standard_normal((M, N)).astype(np.float32)).to(torch.bfloat16)
        self.offset, self.ldc = offset, N + gap if ldc is None else ldc
        self.dev = {n: torch.from_numpy(getattr(self, n)).cuda() for n in ("a", "w", "sa", "sw")}

    def run(self, ssd, bf16=True, add=False, in_place=False):
        M, N = self.M, self.N
        ldc = self.ldc
        dtype = torch.bfloat16 if bf16 else torch.float32
        buf = torch.full((M * ldc + self.offset,), 7.0, dtype=dtype, device="cuda")
        c = buf[self.offset:]
        x, ldadd = None, 0
        if in_place:
            c.view(M, ldc)[:, :N] = self.add.cuda()
            x, ldadd = c, ldc
        elif add:
            x, ldadd = self.add.cuda(), N
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        ssd.ssd_scaled_matmul(M, N, self.K, self.dev["a"], self.lda, self.dev["sa"], self.ldas,
                              self.dev["w"], self.ldw, self.dev["sw"], self.ldws, x, ldadd, c, ldc, st)
        torch.cuda.synchronize()
        assert st.item() == 0
        out = c.view(M, ldc)
        assert (out[:, N:] == 7.0).all() and (buf[:self.offset] == 7.0).all()
        return out[:, :N].double().cpu().numpy()

    def check(self, ssd, bf16=True, add=False, in_place=False):
        got = self.run(ssd, bf16, add, in_place)
        a, w = oc.TABLE[self.a[:, :self.K]], oc.TABLE[self.w[:, :self.K]]
        want, mag = oq.matmul(a, self.sa[:, :self.M].astype(np.float64), w,
                              self.sw.astype(np.float64)[:, :up(self.N, 128) // 128],
                              self.add.double().numpy() if add or in_place else None)
        tol = (132 + len(self.sa)) * 2.0 ** -23 * mag + np.abs(want) * 2.0 ** (-8 if bf16 else -24)
        assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("M", [1, 2, 8, 15, 16, 17, 32, 33, 64, 65, 128, 129, 200, 300])
@pytest.mark.parametrize("N,K", [(64, 64), (128, 128), (129, 300), (1000, 2050)])
def test_sizes(ssd, M, N, K):
    c = Case(M, N, K, M * N + K)
    c.check(ssd, True)
    c.check(ssd, False, add=True)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (3, 2, 16), (70, 1, 5), (129, 65, 17), (5, 700, 12288),
                                   (130, 70, 8200), (64, 129, 4097)])
def test_small_and_long(ssd, M, N, K):
    Case(M, N, K, 5).check(ssd, False)


@pytest.mark.parametrize("M,N,K", [(8, 6144, 4096), (16, 20011, 1024), (50, 9000, 640), (200, 5000, 2050),
                                   (1024, 4096, 1000), (4000, 4100, 300), (513, 12000, 130),
                                   (2500, 333, 1300), (1111, 2300, 4096)])
@pytest.mark.parametrize("bf16", [False, True])
def test_large(ssd, M, N, K, bf16):
    Case(M, N, K, 7).check(ssd, bf16, add=bf16)


@pytest.mark.parametrize("M", [5, 40, 150, 3000])
@pytest.mark.parametrize("gap,offset", [(0, 0), (16, 1), (32, 2), (48, 4)])
def test_alignment_and_in_place(ssd, M, gap, offset):
    """C and add at any alignment to their elements; C added to."""
    c = Case(M, 2600, 256, 11, gap, offset)
    c.check(ssd, True, in_place=True)
    c.check(ssd, False)


@pytest.mark.parametrize("M", [20, 130, 600, 3000])
@pytest.mark.parametrize("N", [1003, 1540, 2494])
def test_rows_on_16_bytes_that_end_inside_of_16(ssd, M, N):
    c = Case(M, N, 400, 19, ldc=N + 8 - N % 8)
    c.check(ssd, True)
    c.check(ssd, True, in_place=True)
    c.check(ssd, False, add=True)


@pytest.mark.parametrize("M,N,K", [(100, 259, 140), (600, 1000, 300), (3000, 2501, 260)])
@pytest.mark.parametrize("more,offset", [(1, 0), (3, 1), (2, 3), (5, 0), (4, 2), (6, 5)])
def test_rows_that_begin_anywhere(ssd, M, N, K, more, offset):
    c = Case(M, N, K, 23, offset=offset, ldc=N + more)
    c.check(ssd, True)
    c.check(ssd, True, add=True)
    c.check(ssd, True, in_place=True)
    c.check(ssd, False)
    c.check(ssd, False, add=True)


def test_offsets_beyond_32_bits(ssd):
    """More than 2^31 entries of C, and of A: the last rows and columns as in a small product."""
    for M, N, K in ((40000, 60000, 128), (20, 1 << 25, 256), (1 << 24, 136, 144)):
        ld = up(K, 16)
        gen = torch.Generator("cuda").manual_seed(M)
        rows = lambda n: torch.randint(0, 0x60, (n, ld), generator=gen, device="cuda",  # noqa: E731
                                       dtype=torch.uint8)
        a, w, C = rows(M), rows(N), up(K, 128) // 128
        sa = torch.rand((C, M), generator=gen, device="cuda") + 0.5
        sw = torch.rand((C, up(N, 128) // 128), generator=gen, device="cuda") + 0.5
        c, st = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ssd.ssd_scaled_matmul(M, N, K, a, ld, sa, M, w, ld, sw, sw.shape[1], None, 0, c, N, st)
        torch.cuda.synchronize()
        assert st.item() == 0
        for i in (slice(0, 3), slice(M // 2, M // 2 + 3), slice(M - 3, M)):
            for j0 in (0, N // 2 // 128 * 128, (N - 1) // 128 * 128):
                j = slice(j0, min(N, j0 + 128))
                x, y = (oc.TABLE[t.cpu().numpy()[:, :K]] for t in (a[i], w[j]))
                want, mag = oq.matmul(x, sa[:, i].double().cpu().numpy(), y,
                                      sw[:, j0 // 128:j0 // 128 + 1].double().cpu().numpy())
                got = c[i, j].double().cpu().numpy()
                assert (np.abs(got - want) <= (132 + C) * 2.0 ** -23 * mag + 2.0 ** -8 * np.abs(want)).all()
        del a, w, c, sa, sw


@pytest.mark.parametrize("M,N,K", [(3, 200, 900), (40, 300, 300), (200, 520, 300), (4000, 4100, 140)])
def test_nan_stays_in_its_row_or_column(ssd, M, N, K):
    c = Case(M, N, K, 13)
    want = c.run(ssd)
    m, n = M - 2, N - 3
    c.dev["a"][m, K - 1] = 0x7f
    c.dev["w"][n, K // 2] = 0xff
    got = c.run(ssd)
    nan = np.zeros((M, N), bool)
    nan[m], nan[:, n] = True, True
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (16, 512, 4096), (200, 5000, 300), (2000, 4100, 600)])
def test_same_bits_again(ssd, M, N, K):
    """Nothing depends on the order of arrival, or on what ran before."""
    c = Case(M, N, K, 17)
    first = c.run(ssd, False)
    for _ in range(3):
        assert np.array_equal(c.run(ssd, False), first)


def test_quantised_inputs_in_a_graph(ssd):
    """Rows and a weight through ssd_quantize and the product, captured and replayed on new rows, and
    two graphs at once on streams of their own: within e4m3's error of the product of the values."""
    M, N, K = 24, 640, 1000
    g = torch.Generator("cuda").manual_seed(3)
    w = torch.randn((N, K), generator=g, device="cuda") * K ** -0.5
    wq, ws = torch.zeros((N, 1008), dtype=torch.uint8, device="cuda"), torch.zeros((8, 5), device="cuda")
    ssd.ssd_quantize(N, K, 128, w, K, wq, 1008, ws, 5)
    work = []
    for i in range(2):
        x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
        q, s = torch.zeros((M, 1008), dtype=torch.uint8, device="cuda"), torch.zeros((8, M), device="cuda")
        c, st = torch.zeros((M, N), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

        def step():
            ssd.ssd_quantize(M, K, 1, x, K, q, 1008, s, M)
            ssd.ssd_scaled_matmul(M, N, K, q, 1008, s, M, wq, 1008, ws, 5, None, 0, c, N, st)

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        x.normal_(generator=g)
        work.append((x, c, st, graph, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, c, st, graph, stream in work:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for x, c, st, graph, stream in work:
        want = x.double() @ w.double().t()
        # each factor is off by at most 2^-4 of itself, 2^-4 / sqrt 3 in the mean of squares
        assert st.item() == 0
        assert (c.double() - want).norm() <= 2 * 2 ** 0.5 * 2.0 ** -4 / 3 ** 0.5 * want.norm()


def test_no_rows(ssd):
    """An empty product does nothing."""
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    t = torch.zeros((1, 16), dtype=torch.uint8, device="cuda")
    c = torch.full((4,), 3.0, device="cuda")
    ssd.ssd_scaled_matmul(0, 4, 16, t, 16, c, 4, t, 16, c, 4, None, 0, c, 4, st)
    torch.cuda.synchronize()
    assert st.item() == 0 and (c == 3.0).all()


def test_products_at_once(ssd):
    """Products of every kernel on two streams give what each gives alone."""
    def call(c, out, st, stream=None):
        ssd.ssd_scaled_matmul(c.M, c.N, c.K, c.dev["a"], c.lda, c.dev["sa"], c.ldas, c.dev["w"], c.ldw,
                              c.dev["sw"], c.ldws, None, 0, out, c.N, st, stream=stream)

    cases = [Case(M, N, 2100, M) for M, N in ((5, 1500), (40, 3000), (60, 300), (200, 1000), (1500, 2049), (2100, 2304))]
    st, streams = torch.zeros(1, dtype=torch.int32, device="cuda"), [torch.cuda.Stream() for _ in range(2)]
    out = [torch.zeros((c.M, c.N), dtype=torch.bfloat16, device="cuda") for c in cases]
    alone = []
    for c, o in zip(cases, out):
        call(c, o, st)
        torch.cuda.synchronize()
        alone.append(o.clone())
        o.zero_()
    torch.cuda.synchronize()
    for _ in range(10):
        for i, (c, o) in enumerate(zip(cases, out)):
            call(c, o, st, streams[i % 2])
    torch.cuda.synchronize()
    assert st.item() == 0
    for o, a in zip(out, alone):
        assert torch.equal(o.view(torch.int16), a.view(torch.int16))
