"""Products of few rows whose waits run out, without a fault: with ssd_set_barrier_shortfall(1) the
epilogue waits for an arrival that nothing makes, and every wait gives up after the polls that
ssd_set_wait_limit allows.  C is left as it was where its sums are not known, whether a tile's blocks
are cut over a cluster or not, and the next call is right."""
import pytest
import torch

from tests.test_gpu_scaled_matmul import Case

pytestmark = pytest.mark.gpu

SSD_ERR_TIMEOUT = 5
# rows; cut over eight, four and two CTAs, and not cut
SIZES = [(3, 100, 2048), (8, 6144, 4096), (16, 12000, 3200), (30, 700, 2050), (50, 1000, 4096), (16, 20011, 300),
         (60, 40000, 260)]


@pytest.fixture(scope="module")
def ssd():
    import paper_2606_20543_gb300 as m
    from paper_2606_20543_gb300 import build
    build.build()
    m.load()
    return m


@pytest.fixture(autouse=True)
def limits(ssd):
    yield
    ssd.ssd_set_barrier_shortfall(0)
    ssd.ssd_set_wait_limit(0)


def call(ssd, c):
    out = torch.full((c.M, c.N), 7.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ssd.ssd_scaled_matmul(c.M, c.N, c.K, c.dev["a"], c.lda, c.dev["sa"], c.ldas, c.dev["w"], c.ldw, c.dev["sw"],
                          c.ldws, None, 0, out, c.N, st)
    torch.cuda.synchronize()
    return out, int(st.item())


@pytest.mark.parametrize("M,N,K", SIZES)
def test_a_wait_that_runs_out_leaves_c(ssd, M, N, K):
    c = Case(M, N, K, 31)
    want, st = call(ssd, c)
    assert st == 0
    ssd.ssd_set_wait_limit(1 << 12)
    ssd.ssd_set_barrier_shortfall(1)
    out, st = call(ssd, c)
    assert st == SSD_ERR_TIMEOUT and (out == 7.0).all()
    ssd.ssd_set_barrier_shortfall(0)
    ssd.ssd_set_wait_limit(0)
    out, st = call(ssd, c)
    assert st == 0 and torch.equal(out, want)


@pytest.mark.parametrize("limit", [1, 4, 64])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_short_limits_leave_c_or_give_it_right(ssd, M, N, K, limit):
    """Whatever gives up, an entry is left or right, and nothing stays in flight."""
    c = Case(M, N, K, 32)
    want, st = call(ssd, c)
    assert st == 0 and not (want == 7.0).any()
    for _ in range(4):
        ssd.ssd_set_wait_limit(limit)
        out, st = call(ssd, c)
        ssd.ssd_set_wait_limit(0)
        left = out == 7.0
        assert st == SSD_ERR_TIMEOUT if left.any() else st in (0, SSD_ERR_TIMEOUT)
        assert torch.equal(out[~left], want[~left])
        out, st = call(ssd, c)
        assert st == 0 and torch.equal(out, want)
