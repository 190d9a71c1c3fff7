"""Host-side argument checks of the paged cache and the sampler: codes come back
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


def test_plan(lib):
    so = lib.load()
    g = ctypes.byref(lib.grid(16, 16, 32))

    def call(grid=g, B=2, block=16, M=8, N=4, cache=F, new=F, held=F, ring=F, R=64, head=F,
             tail=F, nxt=F + 64, table=F, nb=F + 64, slots=F, pos=F, st=F):
        return so.ssd_cache_plan(grid, B, block, M, N, cache, new, held, ring, R, head, tail, nxt,
                                 table, nb, slots, pos, st, None)

    assert call(B=0) == 0
    assert call(B=-1) == call(M=0) == call(N=0) == call(R=0) == call(block=0) == 2
    assert call(block=24) == call(block=256) == call(block=8) == call(M=1 << 30) == 3
    for name in ("cache", "new", "held", "ring", "head", "tail", "nxt", "table", "nb", "slots", "st"):
        assert call(**{name: None}) == 1, name
    assert call(grid=None) == 1 and call(grid=None, pos=None, B=0) == 0
    assert call(nxt=F) == 1 and call(nb=F) == 1 and call(slots=F + 4) == 1


def test_rotary_and_append(lib):
    so = lib.load()
    assert so.ssd_rotary_table(0, 32, F, F, None) == 2
    assert so.ssd_rotary_table(1 << 20, 1 << 12, F, F, None) == 3
    assert so.ssd_rotary_table(16, 32, None, F, None) == 1
    assert so.ssd_rotary_table(16, 32, F, F + 4, None) == 1

    def call(nb=8, block=16, Hkv=2, d=64, k=F, ks=F, sec=(16, 8, 8), npos=9, table=F, B=1, N=4, Hq=4,
             new=F, slots=F, pos=F, q=F, ldq=256, kk=F, ldk=128, v=F, ldv=128, out=F + 4096, st=F):
        c = lib.BlockCache(nb, block, Hkv, d, k, F, ks, F)
        r = lib.Rotary(table, npos, (ctypes.c_int32 * 3)(*sec), 0)
        return so.ssd_cache_append(ctypes.byref(c), ctypes.byref(r), B, N, Hq, new, slots, pos, q,
                                   ldq, kk, ldk, v, ldv, out, st, None)

    assert call(B=0) == 0
    assert call(nb=0) == call(N=0) == call(Hq=3) == call(sec=(16, 8, 9)) == call(npos=0) == 2
    assert call(ldq=248) == call(ldk=120) == call(ldv=132) == call(sec=(40, -8, 0)) == 2
    assert call(block=48) == call(d=96, ldq=384, ldk=192, ldv=192) == call(nb=1 << 28) == 3
    for name in ("k", "ks", "new", "slots", "pos", "q", "kk", "v", "out", "st", "table"):
        assert call(**{name: None}) == 1, name
    assert call(q=F + 8) == call(kk=F + 2) == call(v=F + 4) == call(out=F + 4100) == 1
    assert call(k=F + 8) == call(slots=F + 4) == 1
    assert call(out=F, ldq=264) == 1  # in place only where the rows are packed


def test_attention(lib):
    so = lib.load()
    g = ctypes.byref(lib.grid(16, 16, 32))

    def call(grid=g, nb=8, block=16, Hkv=2, d=64, k=F, B=1, Hq=4, cache=F, nd=F, pos=None, ks=None,
             D=4, table=F, M=4, q=F, scale=0.0, o=F, ws=F, n=1 << 40, st=F):
        c = lib.BlockCache(nb, block, Hkv, d, k, F, F, F)
        return so.ssd_cache_attention(grid, ctypes.byref(c), B, Hq, cache, nd, pos, ks, D, table, M,
                                      q, scale, o, None, ws, n, st, None)

    assert call(B=0) == 0
    assert call(Hq=3) == call(D=0) == call(M=0) == call(B=-1) == 2
    assert call(d=96) == call(block=20) == call(M=1 << 30) == call(B=1 << 16) == 3
    for name in ("grid", "k", "cache", "nd", "table", "q", "o", "st"):
        assert call(**{name: None}) == 1, name
    assert call(q=F + 8) == call(o=F + 2) == call(scale=-1.0) == call(scale=float("nan")) == 1
    need = so.ssd_cache_attention_workspace(1, 4, 2, 64, 4, 1 << 16)
    assert need > 0
    big = dict(M=(1 << 16) // 16, nb=1 << 13)
    assert call(n=need - 1, **big) == call(ws=None, **big) == 7
    assert so.ssd_cache_attention_workspace(0, 4, 2, 64, 4, 64) == 0


def test_sample(lib):
    so = lib.load()

    def call(rows=2, V=100, x=F, bf16=0, ld=100, rng=True, tok=F, st=F, u=F, null=False, **kw):
        p = lib.sampling(**kw)
        r = lib.Rng(0, 0, u)
        return so.ssd_sample(rows, V, x, bf16, ld, None if null else ctypes.byref(p),
                             ctypes.byref(r) if rng else None, tok, None, None, st, None)

    assert call(rows=0, x=None) == 0
    assert call(rows=-1) == call(V=0) == call(ld=99) == 2
    assert call(V=(1 << 20) + 1, ld=1 << 21) == 3
    assert call(null=True) == call(rng=False) == call(x=None) == call(tok=None) == call(st=None) == 1
    assert call(bf16=2) == call(x=F + 2) == call(bf16=1, x=F + 1) == call(u=F + 4) == 1
    for kw in (dict(temperature=-1.0), dict(temperature=float("inf")), dict(top_p=0.0),
               dict(top_p=1.01), dict(min_p=-0.1), dict(min_p=1.5), dict(top_k=-1),
               dict(temperature=float("nan"))):
        assert call(**kw) == 1, kw


def test_python_side_refusals(lib):
    import torch
    k = torch.zeros((4, 2, 16, 64), dtype=torch.uint8)
    s = torch.zeros((4, 2))
    with pytest.raises(ValueError):
        lib.cache(k, k[:2], s, s)
    with pytest.raises(ValueError):
        lib.cache(k.transpose(1, 2), k.transpose(1, 2), s, s)
    with pytest.raises(ValueError):
        lib.cache(k.half(), k.half(), s, s)
    with pytest.raises(ValueError):
        lib.cache(k, k, s, s)  # not on a GPU
    with pytest.raises(ValueError):
        lib.rotary(torch.zeros((5, 32, 2)), (16, 8, 9))
    with pytest.raises(ValueError):
        lib.ssd_sample(1, 4, torch.zeros((1, 4), dtype=torch.float16), 4, lib.sampling(),
                       lib.rng(), None, None, None, None)
