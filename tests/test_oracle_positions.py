"""Pins of the oracle of positions and of the cache in 8 bits (oracle/positions.py), and of the frequencies. No GPU."""
import numpy as np
import pytest
import torch

import paper_2503_05096_amd as pkg
from oracle import positions as P


def test_e4m3_codes_and_rounding_are_the_formats():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(P.E4M3, codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(0, 30, 4000), rng.normal(0, 2e-3, 4000), np.arange(-448, 449) / 2.0 ** rng.integers(0, 12, 897),
                        (P.E4M3[:0x7e] + P.E4M3[1:0x7f]) / 2, [0.0, -0.0, 448.0, -448.0, 463.0]])
    x = np.clip(x, -448, 463).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(P.to_e4m3(x), want)
    assert np.array_equal(P.to_e4m3([np.inf, -np.inf, np.nan]) & 0x7f, [0x7f] * 3)


def test_a_turn_by_hand():
    # position 3, frequency pi / 6: a quarter turn, (a, b) -> (-b, a)
    f = np.array([np.pi / 6, 0.0], np.float32)
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0, 8.0]]], np.float32)
    y = P.rope(x, f, [4], [0], dtype="f32")
    assert np.allclose(y[0, 0], [-3, 2, 1, 4, 9, 8], atol=1e-6)
    y = P.rope(x, f, [4], [0], dtype="f32", interleaved=True, attn_factor=2.0)
    assert np.allclose(y[0, 0], [-4, 2, 6, 8, 9, 8], atol=1e-6)


def test_positions_of_a_tree():
    # two requests: root with children 1, 2; 3 under 1; a chain of two
    parents = [0, 0, 0, 1, 7, -3]
    assert P.row_positions([10, 5], [3, 1], parents) == [(6, 0, 6), (7, 0, 7), (7, 0, 8), (8, 0, 9), (3, 1, 3), (4, 1, 4)]


def test_turning_keeps_lengths_and_angles_add_up():
    rng = np.random.default_rng(1)
    x, f = rng.normal(size=(6, 2, 16)).astype(np.float32), (10000.0 ** (-np.arange(8) / 8)).astype(np.float32)
    y = P.rope(x, f, [200006], [5], dtype="f32")
    assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x.astype(np.float64), axis=-1), rtol=1e-12)
    same = np.repeat(x[:1], 6, axis=0)
    y = P.rope(same, f, [200006], [5], dtype="f32")                 # scores depend on distances alone
    assert np.allclose((y[1] * y[3]).sum(-1), (y[2] * y[4]).sum(-1), rtol=1e-9)


@pytest.mark.parametrize("most,scale", [(448.0, 1.0), (448.0 * (1 + 2.0 ** -40), 2.0), (447.0, 1.0), (224.0, 0.5), (224.01, 1.0),
                                        (3.0, 2.0 ** -7), (0.0, 2.0 ** -100), (1e-300, 2.0 ** -100), (3.4e38, 2.0 ** 120)])
def test_scales(most, scale):
    assert P.scale_for(most * most) == scale


def test_append_scaled_by_hand():
    """One request, one head of one channel pair: a page with two kept tokens, then a louder one."""
    pages = np.zeros((2, 1, 16, 8), np.uint8)
    pages[1, 0, 0], pages[1, 0, 1] = P.to_e4m3(100.0), P.to_e4m3(2.0 ** -9)
    scales = np.array([[9.0], [0.25]])
    k = np.zeros((1, 1, 8), np.float32)
    k[0, 0] = [300, -300, 1, 0, 0, 0, 0, 0]
    kp, vp, ks, vs = P.append_scaled(k, k / 100, None, pages, pages, scales, scales, [[1]], [3], [0], dtype="f32")
    assert ks[1, 0] == 1.0 and ks[0, 0] == 9.0 and vs[1, 0] == 0.25        # 300 does not fit 448 / 4; 3 does
    assert np.array_equal(P.E4M3[kp[1, 0, 0]], [24.0] * 8)                  # 100, halfway between 96 and 104, is stored as 96
    assert np.array_equal(P.E4M3[kp[1, 0, 1]], [0.0] * 8)                   # 2^-11: a quarter of the least code
    assert np.array_equal(P.E4M3[kp[1, 0, 2]][:3], [288.0, -288.0, 1.0]) and np.array_equal(vp[1, 0, :2], pages[1, 0, :2])
    assert np.array_equal(P.E4M3[vp[1, 0, 2]][:3], [12.0, -12.0, 0.0390625])


def test_frequencies():
    f, gain = pkg.rope_frequencies(8, base=10000.0)
    assert f.dtype == torch.float32 and gain == 1.0 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001]), rtol=1e-7)
    assert torch.equal(pkg.rope_frequencies(8, scaling={"kind": "linear", "factor": 4})[0], f / 4)
    g, _ = pkg.rope_frequencies(8, scaling={"kind": "base", "factor": 4})
    assert g[0] == 1 and abs(float(g[-1]) / 0.00025 - 1) < 1e-6
    g, gain = pkg.rope_frequencies(128, base=500000.0, scaling={"kind": "wavelengths", "factor": 8, "trained": 8192})
    h = pkg.rope_frequencies(128, base=500000.0)[0]
    turns = 8192 * h.double() / (2 * np.pi)
    assert gain == 1.0 and torch.equal(g[turns > 4], h[turns > 4]) and torch.allclose(g[turns < 1], h[turns < 1] / 8, rtol=1e-6)
    assert bool(((g <= h) & (g >= h / 8.001)).all()) and bool((g[1:] < g[:-1]).all())
    g, gain = pkg.rope_frequencies(64, scaling={"kind": "ramp", "factor": 16, "trained": 4096})
    h = pkg.rope_frequencies(64)[0]
    assert abs(gain - (0.1 * np.log(16) + 1)) < 1e-12 and g[0] == h[0] and abs(float(g[-1] / h[-1]) * 16 - 1) < 1e-6
    for kw in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, base=0), dict(rot_dim=8, scaling={"kind": "other"}),
               dict(rot_dim=8, scaling={"kind": "linear", "factor": 0}), dict(rot_dim=8, scaling={"kind": "linear", "factor": 2, "x": 1}),
               dict(rot_dim=2, scaling={"kind": "base", "factor": 2}),
               dict(rot_dim=8, scaling={"kind": "wavelengths", "factor": 2, "trained": 100, "low": 4, "high": 4})):
        with pytest.raises(ValueError):
            pkg.rope_frequencies(**kw)


def test_compact_path_by_hand():
    """Nodes 2 and 3 of 4 drafts accepted; base 14: the root in slot 14 of the first page, node 1 in slot 15, the rest in the second."""
    pages, scales = np.zeros((2, 1, 16, 8), np.uint8), np.array([[1.0], [4.0]])
    for slot in range(16):
        pages[0, 0, slot] = P.to_e4m3(float(slot + 1))
        pages[1, 0, slot] = P.to_e4m3(32.0 + 4 * slot)
    p, s = P.compact_path_scaled(pages, scales, [[0, 1]], [19], [4], [[2, 3, -1, -1, -1]], [2])
    assert s.tolist() == [[4.0], [4.0]]
    assert np.array_equal(P.E4M3[p[0, 0, 14]], [3.75] * 8) and np.array_equal(P.E4M3[p[0, 0, 15]], [32.0] * 8)
    assert np.array_equal(P.E4M3[p[1, 0, 0]], [36.0] * 8)
