"""The buffers that PagedDecode keeps, on the CPU: their sizes are host code."""
import os
import shutil

import pytest


@pytest.fixture(scope="module")
def ssd():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2606_20543_gb300 import build
    build.build()
    import paper_2606_20543_gb300 as m
    m.load()
    return m


@pytest.fixture(autouse=True)
def sharing(ssd):
    yield
    ssd.load().ssd_set_cache_sharing(0)


def make(groups, max_shared, B=4, max_blocks=200):
    """A decoder without the tensors that only a GPU fills."""
    from paper_2606_20543_gb300.decode import PagedDecode
    dec = PagedDecode.__new__(PagedDecode)
    dec.__dict__.update(B=B, Hq=8, Hkv=2, d=128, block=16, max_blocks=max_blocks, device="cpu", groups=groups,
                        max_shared=max_shared, _ws={}, _outgrown=[])
    return dec


def test_the_workspace_follows_the_switch_whoever_sets_it(ssd):
    so, dec = ssd.load(), make(2, 90)
    need = lambda: so.ssd_cache_attention_shared_workspace(4, 2, 8, 2, 128, 1, 3200, 1440)  # noqa: E731
    assert ssd.ssd_get_cache_sharing() == 0
    sizes = []
    for how in (2, 1, 0, 1):
        assert so.ssd_set_cache_sharing(how) == 0  # (as a caller of the C library does)
        assert ssd.ssd_get_cache_sharing() == how
        ws, n = dec._workspace(1)
        assert n >= need() and n == ws.numel()
        sizes.append(need())
    assert sizes[1] > sizes[0]
