"""A host thread that has made no CUDA call of its own calls the entry points that copy by TMA: its
first call is as good as any other thread's (a tensor map is encoded by the driver, which wants a
current context, and a thread gets one with its first call of the CUDA runtime)."""
import threading

import pytest
import torch

from tests.test_gpu_cache_attention import i32, ssd  # noqa: F401

pytestmark = pytest.mark.gpu


def in_fresh_thread(call, out):
    """call() here, then in a thread of its own: the same results in `out`."""
    call()
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    for x in out:
        x.zero_()
    torch.cuda.synchronize()
    errors = []

    def work():
        try:
            call()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for x, y in zip(out, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("D", [1, 24])
def test_cache_attention(ssd, D):  # noqa: F811
    gen = torch.Generator("cuda").manual_seed(D)
    Hq, Hkv, d, block, cache, M = 4, 2, 128, 16, 40, 10000
    pool = -(-(cache + D) // block)
    k, v = (torch.randn((pool, Hkv, block, d), generator=gen, device="cuda").to(torch.float8_e4m3fn)
            for _ in range(2))
    ks, vs = (torch.ones((pool, Hkv), device="cuda") for _ in range(2))
    c, g = ssd.cache(k, v, ks, vs), ssd.grid(16, 16, 0)
    table = torch.full((1, M), -1, dtype=torch.int32, device="cuda")
    table[0, :pool] = torch.arange(pool, device="cuda")
    q = torch.randn((1, D, Hq, d), generator=gen, device="cuda").to(torch.bfloat16)
    o, st, cl, nd = torch.zeros_like(q), i32([0]), i32([cache]), i32([D])
    n = ssd.ssd_cache_attention_workspace(1, Hq, Hkv, d, D, M * block)
    ws = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    in_fresh_thread(lambda: ssd.ssd_cache_attention(g, c, 1, Hq, cl, nd, None, None, D, table, M, q, 0.0,
                                                    o, None, ws, n, st, stream=stream), [o, st])


@pytest.mark.parametrize("D,Hq,Hkv", [(16, 4, 4), (3, 520, 4)])
def test_verify_attention(ssd, D, Hq, Hkv):  # noqa: F811
    """Both kernels."""
    gen = torch.Generator("cuda").manual_seed(Hq)
    d, L, cache, G = 128, 128, 40, Hq // Hkv
    assert D * G <= 512
    q = torch.randn((1, D, Hq, d), generator=gen, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((1, Hkv, L, d), generator=gen, device="cuda").to(torch.bfloat16)
            for _ in range(2))
    g, o, st, cl, nd = ssd.grid(16, 16, 0), torch.zeros_like(q), i32([0]), i32([cache]), i32([D])
    pos = i32([list(range(cache, cache + D))])
    n = ssd.ssd_verify_attention_workspace(1, Hq, Hkv, d, D, L)
    ws = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    in_fresh_thread(lambda: ssd.ssd_verify_attention(g, 1, Hq, Hkv, d, cl, nd, pos, D, L, q, k, v, 0.0, o,
                                                     None, ws, n, st, stream=stream), [o, st])


def test_predictor(ssd):  # noqa: F811
    from tests.test_gpu_predictor import _bf_dev, _case
    rows, d, m, V = 16, 256, 512, 2048
    w, g1, g2 = _case(31, rows, d, m, V)
    dev = {k: _bf_dev(x) for k, x in w.items()}
    dev["g1"], dev["g2"] = torch.from_numpy(g1).cuda(), torch.from_numpy(g2).cuda()
    n = ssd.ssd_draft_predict_workspace(rows, d, m, V)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    tok, st = torch.zeros(rows, dtype=torch.int32, device="cuda"), i32([0])
    hid = torch.zeros((rows, d), device="cuda")
    stream = torch.cuda.Stream()
    in_fresh_thread(lambda: ssd.ssd_draft_predict(rows, d, m, V, dev["z"], dev["w0"], dev["w1"], dev["w3"],
                                                  dev["w2"], dev["g1"], dev["g2"], dev["wh"], 1e-6, tok,
                                                  hid, ws, n, st, stream=stream), [tok, hid, st])
