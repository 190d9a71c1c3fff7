"""Host-side argument checks of the 8-bit products and of the head norms: codes come back
without touching a GPU (every pointer below is a fake that is never read)."""
import ctypes
import shutil
import os

import pytest

F = 0x1000


@pytest.fixture(scope="module")
def lib():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2606_20543_gb300 import build
    build.build()
    import paper_2606_20543_gb300 as ssd
    return ssd


def test_quantize(lib):
    so = lib.load()

    def call(rows=200, K=300, block=1, x=F, bf16=1, ldx=304, out=F, ldo=304, scale=F, lds=200):
        return so.ssd_quantize(rows, K, block, x, bf16, ldx, out, ldo, scale, lds, None)

    assert call(rows=0, lds=0) == 0
    assert call(rows=-1) == call(K=0) == call(block=0) == call(ldx=296) == call(ldo=288) == 2
    assert call(ldx=308) == call(ldo=312) == call(lds=199) == call(block=128, lds=1) == 2
    assert call(block=2) == call(block=64) == call(K=1 << 24, ldx=1 << 24, ldo=1 << 24) == 3
    for name in ("x", "out", "scale"):
        assert call(**{name: None}) == 1, name
    assert call(bf16=2) == call(x=F + 8) == call(out=F + 8) == call(scale=F + 2) == 1


def test_matmul(lib):
    so = lib.load()

    def call(M=5, N=200, K=300, a=F, lda=304, sa=F, ldas=5, w=F, ldw=304, sw=F, ldws=2, add=None, ldadd=0,
             c=F, bf16=1, ldc=200, st=F):
        return so.ssd_scaled_matmul(M, N, K, a, lda, sa, ldas, w, ldw, sw, ldws, add, ldadd, c, bf16, ldc,
                                    st, None)

    assert call(M=0) == 0
    assert call(M=-1) == call(N=0) == call(K=0) == call(lda=288) == call(ldw=288) == call(ldc=199) == 2
    assert call(ldas=4) == call(ldws=1) == call(lda=312) == call(ldw=308) == call(add=F, ldadd=199) == 2
    big = 1 << 30
    assert call(M=big, ldas=big, N=big, ldc=big, ldws=big) == call(lda=1 << 40) == 3
    for name in ("a", "w", "sa", "sw", "c", "st"):
        assert call(**{name: None}) == 1, name
    assert call(a=F + 8) == call(w=F + 8) == call(sa=F + 2) == call(sw=F + 1) == call(c=F + 1) == 1
    assert call(bf16=0, c=F + 2) == call(bf16=2) == call(add=F + 1, ldadd=200) == 1


def test_append_norm(lib):
    so = lib.load()

    def call(kind=1, eps=1e-6, gains=(F, F, F, F), heads=(0, 0), Hq=4, B=1, null=False, d=64):
        c = lib.BlockCache(8, 16, 2, d, F, F, F, F)
        r = lib.Rotary(F, 9, (ctypes.c_int32 * 3)(16, 8, 8), 0)
        n = lib.HeadNorm(kind, eps, *gains, *heads)
        return so.ssd_cache_append_norm(ctypes.byref(c), ctypes.byref(r),
                                        None if null else ctypes.byref(n), B, 4, Hq, F, F, F, F, 256,
                                        F, 128, F, 128, F + 4096, F, None)

    assert call(B=0) == call(B=0, kind=2, heads=(4, 2), gains=(None, F, F, None)) == 0
    assert call(null=True) == call(kind=0) == call(kind=3) == 1
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert call(eps=eps) == 1
    assert call(heads=(2, 0)) == call(heads=(0, 4)) == call(heads=(-1, 0)) == call(Hq=3) == 2
    for i in range(4):
        assert call(gains=[F + 4 if i == j else F for j in range(4)]) == 1


def test_shared_attention(lib):
    so = lib.load()
    g = ctypes.byref(lib.grid(16, 16, 32))

    def call(grid=g, nb=8, block=16, Hkv=2, d=64, k=F, B=4, groups=2, start=F, shared=F, most=3, Hq=4, cache=F,
             nd=F, D=4, table=F, M=4, q=F, scale=0.0, o=F, ws=F, n=1 << 40, st=F):
        c = lib.BlockCache(nb, block, Hkv, d, k, F, F, F)
        return so.ssd_cache_attention_shared(grid, ctypes.byref(c), B, groups, start, shared, most, Hq, cache, nd,
                                             None, None, D, table, M, q, scale, o, None, ws, n, st, None)

    assert call(B=0) == 0
    assert call(groups=0) == call(most=-1) == call(most=5) == call(Hq=3) == call(D=0) == call(B=-1) == 2
    assert call(groups=70000) == call(d=96) == call(B=1 << 16) == call(M=1 << 30) == 3
    for name in ("grid", "k", "start", "shared", "cache", "nd", "table", "q", "o", "st"):
        assert call(**{name: None}) == 1, name
    assert call(q=F + 8) == call(o=F + 2) == call(scale=-1.0) == 1
    assert so.ssd_set_cache_sharing(3) == so.ssd_set_cache_sharing(-1) == 1
    assert so.ssd_set_cache_sharing(1) == 0
    try:
        need = so.ssd_cache_attention_shared_workspace(4, 2, 4, 2, 64, 4, 64, 48)
        assert need > 0 and call(n=need - 1) == call(ws=None) == 7 and call(ws=F + 8) == 1
    finally:
        assert so.ssd_set_cache_sharing(0) == 0
    assert so.ssd_cache_attention_shared_workspace(4, 0, 4, 2, 64, 4, 64, 48) == 0
    assert so.ssd_cache_attention_shared_workspace(4, 2, 4, 2, 64, 4, 64, 65) == 0
    # many sequences over a long prompt share by themselves, few do not
    few = so.ssd_cache_attention_shared_workspace(2, 1, 32, 8, 128, 1, 8192, 8000)
    assert few == so.ssd_cache_attention_workspace(2, 32, 8, 128, 1, 8192)
    many = so.ssd_cache_attention_shared_workspace(64, 1, 32, 8, 128, 1, 8192, 8000)
    assert many != so.ssd_cache_attention_workspace(64, 32, 8, 128, 1, 8192)


def test_python_side_refusals(lib):
    import torch
    g = torch.ones(64)
    with pytest.raises(ValueError):
        lib.head_norm("rms", 1e-6, g)  # not on a GPU
    with pytest.raises(ValueError):
        lib.head_norm("rms", 1e-6, g.double())
    with pytest.raises(ValueError):
        lib.head_norm("rms", 1e-6, torch.ones(4, 64), g)
    with pytest.raises(ValueError):
        lib.head_norm("rms", 1e-6, torch.ones(64, 2)[:, 0])
    with pytest.raises(ValueError):
        lib.head_norm("rms", 1e-6, None, g, None, torch.ones(128))
    n = lib.head_norm("layer", 1e-6)
    assert (n.kind, n.q_heads, n.k_heads) == (2, 0, 0)
    n.d = 128
    with pytest.raises(ValueError):
        lib.ssd_cache_append_norm(lib.BlockCache(8, 16, 2, 64, F, F, F, F), lib.Rotary(), n, 1, 1, 4,
                                  *[None] * 12)
    with pytest.raises(ValueError):
        lib.ssd_scaled_matmul(1, 1, 16, None, 16, None, 1, None, 16, None, 1, torch.zeros(1), 1, None, 1,
                              None)
    with pytest.raises(ValueError):
        lib.ssd_scaled_matmul(1, 1, 16, torch.zeros(16), 16, None, 1, None, 16, None, 1, None, 1, None, 1,
                              None)
    with pytest.raises(ValueError):
        lib.ssd_quantize(1, 8, 1, torch.zeros((1, 8), dtype=torch.float16), 8, None, 16, None, 1)
