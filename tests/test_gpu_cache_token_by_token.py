"""The same tokens appended one by one and as one prompt.  Both end with the scale of the largest
value, exactly.  An entry of the prompt was rounded once; one of a token by itself once more for
every later token that raised its block's scale, each time by at most half an e4m3 step: 2^-4 of
the value as it then is, or 2^-10 of the scale where the value is below e4m3's normal range.  The
products that are rounded carry float32's errors (2^-21 covers them)."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.test_gpu_cache_attention import i32, ssd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block,d,L", [(16, 64, 40), (64, 128, 130), (128, 64, 128)])
def test_one_by_one_and_as_a_prompt(ssd, block, d, L):  # noqa: F811
    from paper_2606_20543_gb300.decode import PagedDecode
    Hkv, M = 2, -(-L // block)
    gen = torch.Generator("cuda").manual_seed(block)
    x = torch.randn((L, Hkv, d), generator=gen, device="cuda")
    x *= torch.exp(0.7 * torch.randn((L, Hkv, 1), generator=gen, device="cuda"))
    x = x.to(torch.bfloat16).view(L, Hkv * d)
    got = []
    for N in (1, L):
        # (no frequency: keys are not turned, so both are exact before they are rounded)
        dec = PagedDecode(ssd.grid(1, 1, L), 1, Hkv, Hkv, d, M, block, M, N,
                          torch.zeros(d // 2, device="cuda"), (d // 2, 0, 0))
        for i in range(0, L, N):
            dec.plan(i32([N]), N)
            dec.attend(0, x[i:i + N], x[i:i + N], x[i:i + N])
            dec.advance()
        assert int(dec.status.item()) == 0
        t = dec.block_table[0].cpu().numpy()
        for code, scale in ((dec.k, dec.k_scale), (dec.v, dec.v_scale)):
            c = oc.TABLE[code[0].view(torch.uint8).cpu().numpy()[t]]          # [M, Hkv, block, d]
            got.append((c.transpose(0, 2, 1, 3).reshape(-1, Hkv, d)[:L],
                        scale[0].cpu().numpy()[t]))
    want = x.double().cpu().numpy().reshape(L, Hkv, d)
    top = np.abs(want).max(-1)                                                # [L, Hkv]
    grown = np.zeros((L, Hkv), int)  # roundings after the first
    for i in range(M):
        rows = slice(i * block, min(L, (i + 1) * block))
        run = np.maximum.accumulate(top[rows], 0)
        up = np.zeros(run.shape, int)
        up[1:] = run[1:] > run[:-1]
        grown[rows] = up[::-1].cumsum(0)[::-1] - up
    assert grown.max() >= 2
    for k in range(2):
        (one, s1), (prompt, s2) = got[k], got[2 + k]
        assert np.array_equal(s1, s2)
        s = s1.astype(np.float64)[np.arange(L) // block][:, :, None]
        for value, n in ((prompt * s, np.zeros_like(grown)), (one * s, grown)):
            n = n[:, :, None] + 1
            up = (1 + 2.0 ** -4) ** n
            tol = n * (2.0 ** -4 * up * np.abs(want) + 2.0 ** -10 * s) * (1 + 2.0 ** -21)
            assert np.all(np.abs(value - want) <= tol)
