"""The float64 cache and sampler oracles against what fixes them."""
import numpy as np
import torch

from oracle import cache as oc
from oracle import sample as osm


def test_e4m3_table_and_rounding_match_torch():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, oc.TABLE, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-12, 9, 5001)])
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oc.e4m3_round(x.astype(np.float32).astype(np.float64)), want)


def test_rotation_keeps_lengths_and_relative_positions():
    g = np.random.default_rng(0)
    d, freq = 16, 10000.0 ** (-np.arange(8) / 8)
    x = g.standard_normal((5, 2, d))
    pos = g.integers(0, 50, (5, 3))
    for inter in (False, True):
        y = oc.rotate(x, pos, freq, (2, 3, 3), inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        # a score depends on the difference of the positions on every axis alone
        a = oc.rotate(x[:1], pos[:1], freq, (2, 3, 3), inter)[0, 0]
        b = oc.rotate(x[1:2], pos[1:2], freq, (2, 3, 3), inter)[0, 0]
        a2 = oc.rotate(x[:1], pos[:1] + 7, freq, (2, 3, 3), inter)[0, 0]
        b2 = oc.rotate(x[1:2], pos[1:2] + 7, freq, (2, 3, 3), inter)[0, 0]
        assert np.isclose(a @ b, a2 @ b2)
        assert np.allclose(oc.rotate(x, pos * 0, freq, (2, 3, 3), inter), x)


def test_plan_deals_every_block_once():
    ring = np.array([9, 4, 7, 1, 5, 0, 2])
    table = np.full((3, 4), -1)
    table[0, 0], table[2, :2] = 3, (6, 8)
    t, n, head, slots, pos, served = oc.plan(4, 4, 5, 16, 4, 40, [10, 0, 32], [7, 33, 0], [1, 0, 2],
                                             ring, 6, 13, table)
    assert served.all() and head == 6 + 1 + 3 and list(n) == [2, 3, 2]
    assert list(t[0, :2]) == [3, 2] and list(t[1, :3]) == [9, 4, 7]
    assert slots[0, 5] == 3 * 16 + 15 and slots[0, 6] == 2 * 16 and slots[0, 7] == -1
    assert tuple(pos[1, 4]) == (4, 4, 4) and tuple(pos[1, 5 + 6]) == (5, 6, 7)
    # out of blocks: the second and every later one that wants some go without
    t, n, head, slots, _, served = oc.plan(4, 4, 5, 16, 4, 40, [10, 0, 32], [7, 33, 1], [1, 0, 2],
                                           ring, 6, 9, table)
    assert list(served) == [True, False, False] and head == 7 and (slots[1:] == -1).all()


def test_sampler_law_on_a_small_vocabulary():
    """The share of each token over evenly spread uniforms is its probability
    under the filters, enumerated by hand."""
    x = np.log(np.array([1.0, 4.0, 2.0, 8.0, 1.0, 0.5]))
    u = (np.arange(20000) + 0.5) / 20000

    def law(**kw):
        s = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
        s.update(kw)
        t = [osm.sample_row(x, s["temperature"], s["top_k"], s["top_p"], s["min_p"], v)["tok"]
             for v in u[::10]]
        return np.bincount(t, minlength=6) / len(t)

    assert np.allclose(law(), np.array([1, 4, 2, 8, 1, .5]) / 16.5, atol=1e-3)
    assert np.allclose(law(top_k=2), np.array([0, 4, 0, 8, 0, 0]) / 12, atol=1e-3)
    # mass before: 8 -> 0, 4 -> 8, 2 -> 12, 1 -> 14 of 16.5
    assert np.allclose(law(top_p=0.75), np.array([0, 4, 2, 8, 0, 0]) / 14, atol=1e-3)
    assert np.allclose(law(top_p=0.72), np.array([0, 4, 0, 8, 0, 0]) / 12, atol=1e-3)
    # top-p of what top-k left: 12 * 0.7 = 8.4
    assert np.allclose(law(top_k=3, top_p=0.55), np.array([0, 0, 0, 1, 0, 0]), atol=1e-3)
    assert np.allclose(law(min_p=0.2), np.array([0, 4, 2, 8, 0, 0]) / 14, atol=1e-3)
    # equal logits: the lower index first
    assert osm.sample_row(x, 1.0, 4, 1.0, 0.0, 0.999)["ids"].tolist() == [0, 1, 2, 3]
    assert np.allclose(law(temperature=0.5, top_k=2), np.array([0, 16, 0, 64, 0, 0]) / 80, atol=1e-3)


def test_attention_of_one_key_and_of_none():
    g = np.random.default_rng(1)
    q, k, v = g.standard_normal((2, 4, 8)), g.standard_normal((3, 2, 8)), g.standard_normal((3, 2, 8))
    see = np.array([[False, True, False], [False, False, False]])
    o, lse, _, _, _ = oc.attention(q, k, v, see, 0.5, np.ones((3, 2)))
    assert np.allclose(o[0, 1], v[1, 0]) and np.allclose(o[0, 2], v[1, 1])
    assert (o[1] == 0).all() and (lse[1] == -np.inf).all()
    assert np.isclose(lse[0, 3], 0.5 * q[0, 3] @ k[1, 1])
