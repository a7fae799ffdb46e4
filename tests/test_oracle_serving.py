"""Pins of oracle/serving.py: e4m3 rounding against torch's conversion, the norm and
the scales against closed forms, the product against integers, and the processing of
one row against values worked out by hand."""

import numpy as np
import torch

from oracle import serving


def test_e4m3_rounding_against_torch():
    """Every e4m3 value is a fixed point; random values over the format's range and the
    midpoints between neighbours round as torch's float32 -> e4m3 conversion does."""
    codes = torch.arange(256, dtype=torch.int16).to(torch.uint8)
    values = codes.view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    finite = values[np.isfinite(values)]
    assert np.array_equal(serving.round_e4m3(finite), finite)
    assert finite.max() == serving.E4M3_MAX
    grid = np.unique(finite)
    mid = (grid[1:] + grid[:-1]) / 2
    g = np.random.default_rng(3)
    rnd = np.concatenate([g.uniform(-448, 448, 20000), g.normal(size=20000),
                          np.exp2(g.uniform(-12, 8.8, 20000))]).astype(np.float32)
    x = np.concatenate([mid, rnd]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(serving.round_e4m3(x), want)
    assert serving.round_e4m3(1000.0) == 448.0 and serving.round_e4m3(-1e9) == -448.0


def test_norm_closed_forms():
    """A constant row c: y = w c / sqrt(c^2 + eps).  A row with one entry c of K:
    y = w c sqrt(K) / sqrt(c^2 + K eps)."""
    w = np.linspace(0.5, 2.0, 24)
    y, h = serving.rms_norm(np.full((1, 24), 1.5), np.full((1, 24), 1.5), w, 1e-3)
    assert np.allclose(h, 3.0) and np.allclose(y[0], w * 3.0 / np.sqrt(9.0 + 1e-3), rtol=1e-14)
    x = np.zeros((1, 24))
    x[0, 5] = -2.0
    y, _ = serving.rms_norm(x, None, w, 1e-3)
    assert np.isclose(y[0, 5], -2.0 * w[5] * np.sqrt(24) / np.sqrt(4.0 + 24e-3), rtol=1e-14)
    assert np.all(np.delete(y[0], 5) == 0)


def test_scales_of_ragged_groups():
    y = np.zeros((3, 130))
    y[0, 127], y[0, 128], y[1, 0] = -7.0, 448.0, 3.0
    s = serving.row_scales(y)
    assert s.shape == (3, 2)
    assert s[0, 0] == 7.0 / 448 and s[0, 1] == 1.0 and s[1, 0] == 3.0 / 448
    assert s[2, 0] == 2.0 ** -100 / 448
    w = np.zeros((129, 130))
    w[128, 129], w[5, 6] = 4.48, -448.0
    b = serving.block_scales(w)
    assert b.shape == (2, 2) and b[0, 0] == 1.0 and np.isclose(b[1, 1], 0.01)


def test_scaled_logits_against_integers():
    g = np.random.default_rng(1)
    qa, qw = g.integers(-8, 9, (3, 200)), g.integers(-8, 9, (130, 200))
    sa, sw = 2.0 ** g.integers(-3, 4, (3, 2)), 2.0 ** g.integers(-3, 4, (2, 2))
    got = serving.scaled_logits(qa, sa, qw, sw)
    for i, v in ((0, 0), (1, 127), (2, 128), (2, 129)):
        want = sum(float(sa[i, k // 128] * sw[v // 128, k // 128]) * int(qa[i, k]) * int(qw[v, k])
                   for k in range(200))
        assert got[i, v] == want


def test_processed_row_by_hand():
    """Token 0: generated twice and once on the path; 1: in the prompt, negative logit;
    2: on the path only; 3: biased; 4: masked; 5: untouched."""
    l = [3.0, -1.0, 2.0, 0.5, 9.0, 0.25]
    got = serving.process_row(l, [2, 0, 0, 0, 0, 0], [0, 1, 0, 0, 0, 0], [0, 0, 0, 1.5, 1, 0],
                              (2.0, 0.25, 0.5), [0, 2], [1, 1, 1, 1, 0, 1])
    assert got.tolist() == [1.5 - 0.75 - 0.5, -2.0, 1.0 - 0.25 - 0.5, 2.0, -np.inf, 0.25]
    m, s = serving.row_normaliser(got, 0.5)
    assert m == 2.0
    assert np.isclose(s, sum(np.exp((v - 2.0) / 0.5) for v in got))
    assert serving.row_normaliser(np.full(4, -np.inf), 1.0) == (-np.inf, 0.0)
    assert serving.path_tokens([-1, 0, 1, 0], [9, 4, 5, 6], 2) == [5, 4]
    assert serving.path_tokens([-1, 0, 1, 0], [9, 4, 5, 6], 0) == []
