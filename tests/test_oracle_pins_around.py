"""Pins of the oracle's norm, draws and clipping: hand-worked examples, closed forms, identities and finite differences."""
import math

import numpy as np
import pytest
import torch

from oracle import umas_oracle as orc


def test_norm_by_hand():
    y, inv = orc.rms_norm(np.array([[3.0, 4.0], [0.0, 0.0]]), np.array([2.0, 1.0]), 0.5)
    assert np.allclose(inv, [13.0 ** -0.5, 2.0 ** 0.5]) and np.allclose(y, [[6 / 13 ** 0.5, 4 / 13 ** 0.5], [0, 0]])


def test_norm_backward_by_differences():
    rng = np.random.default_rng(1)
    s, g, v, eps, h = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), 0.1, 1e-5
    f = lambda s, g: (orc.rms_norm(s, g, eps)[0] * v).sum()
    dx, dg = orc.rms_norm_backward(v, s, g, orc.rms_norm(s, g, eps)[1])
    for i in range(3):
        for j in range(7):
            e = np.zeros((3, 7))
            e[i, j] = h
            assert abs((f(s + e, g) - f(s - e, g)) / (2 * h) - dx[i, j]) < 1e-8
    for j in range(7):
        e = np.zeros(7)
        e[j] = h
        assert abs((f(s, g + e) - f(s, g - e)) / (2 * h) - dg[j]) < 1e-8
    # with eps = 0 the norm does not see a row's length: the gradient stands upright on the row
    inv = orc.rms_norm(s, g, 0.0)[1]
    dx, _ = orc.rms_norm_backward(v, s, g, inv)
    assert np.abs((dx * s).sum(1)).max() < 1e-14
    through, _ = orc.rms_norm_backward(v * [[1], [0], [1]], s * [[1], [np.nan], [1]], g, inv, np.ones((3, 7)))
    assert np.allclose(through[0], dx[0] + 1) and (through[1] == 1).all()


def test_numbers_of_8_bits():
    v = orc.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[56] == 1.0 and v[57] == 1.125 and v[126] == 448 and (np.diff(v) > 0).all()
    assert np.array_equal(torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy(), v)


def test_draws_by_hand():
    z = np.log([1.0, 4.0, 2.0, 1.0, 2.0])                            # of 10
    want = lambda u, **s: orc.sample(z, u, **s)[0]
    assert [want(u) for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.79, 0.81, 0.99, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3, 4, 4, 4]
    assert [want(u, top_k=2) for u in (0.0, 0.66, 0.67, 0.99)] == [1, 1, 2, 2]                  # 4 and the first 2
    assert [want(u, top_k=4) for u in (0.0, 0.1, 0.12, 0.99)] == [0, 0, 1, 4]                   # the first of the two ones
    assert [want(u, min_p=0.5) for u in (0.0, 0.49, 0.51, 0.74, 0.76)] == [1, 1, 2, 2, 4]
    assert [want(u, top_p=0.59) for u in (0.0, 0.66, 0.67)] == [1, 1, 2]                        # 4 are too few, 6 enough
    assert [want(u, top_p=0.61) for u in (0.0, 0.76, 0.99)] == [1, 4, 4]
    assert [want(u, top_p=0.0) for u in (0.0, 0.99)] == [1, 1] and want(0.99, temperature=0.0) == 1
    assert [want(u, top_k=3, top_p=0.49) for u in (0.0, 0.99)] == [1, 1]                        # 4 of 8
    assert [want(u, top_k=3, top_p=0.51) for u in (0.0, 0.99)] == [1, 2]
    assert [want(u, temperature=0.5) for u in (0.03, 0.04, 0.65, 0.66, 0.99)] == [0, 1, 1, 2, 4]   # 1 16 4 1 4 of 26
    t, logp, logq = orc.sample(z, 0.7, temperature=0.5, top_k=2)
    assert t == 1 and abs(logp - math.log(0.4)) < 1e-15 and abs(logq - math.log(0.8)) < 1e-15


def test_draws_of_masked_rows():
    inf = math.inf
    assert orc.sample(np.full(3, -inf), 0.5) == (-1, 0.0, 0.0) and orc.sample(np.full(3, np.nan), 0.5) == (-1, 0.0, 0.0)
    assert orc.sample(np.array([-inf, 2.0, np.nan]), 0.99) == (1, 0.0, 0.0)
    t, logp, logq = orc.sample(np.array([1.0, inf, 2.0, inf]), 0.6)
    assert t == 3 and abs(logp + math.log(2)) < 1e-15 and abs(logq + math.log(2)) < 1e-15
    assert orc.sample(np.array([-3e38, -3e38]), 0.6)[0] == 1 and orc.sample(np.array([-0.0, 0.0, -0.0]), 0.5, top_k=2)[0] == 1


def test_draws_follow_the_distribution():
    rng = np.random.default_rng(2)
    z = rng.normal(size=30) * 2
    p = torch.softmax(torch.tensor(z) / 0.8, 0).numpy()
    u = (np.arange(20000) + 0.5) / 20000
    got = np.bincount([orc.sample(z, x, temperature=0.8)[0] for x in u], minlength=30) / 20000
    assert np.abs(got - p).max() <= 1 / 20000 + 1e-12                # one uniform number apart at either end


def test_clipping_by_hand():
    norm, c, bad, out = orc.clip([np.array([3.0]), np.array([[0.0, 4.0]])], 1.0)
    assert (norm, bad) == (5.0, 0) and abs(c - 0.2) < 1e-16 and np.allclose(out[0], 0.6) and np.allclose(out[1], [[0, 0.8]])
    assert orc.clip([np.array([3.0, 4.0])], 5.0)[1] == 1.0 and orc.clip([np.zeros(3)], 1.0)[:2] == (0.0, 1.0)
    with np.errstate(all="ignore"):
        assert orc.clip([np.array([np.inf, 1.0]), np.array([np.nan])], 1.0)[1:3] == (1.0, 2)
