"""Pins of the oracle's largest logits, cross entropy and distillation: hand-worked examples, closed forms, identities and finite differences (none of
them retypes the oracle's formula)."""
import math

import numpy as np
import pytest
import torch

from oracle import umas_oracle as orc


def test_top_logits_by_hand_with_ties_and_gaps():
    # one hidden column of 1: the logits are the rows of W
    W = np.array([[1.0], [3.0], [2.0], [3.0], [-np.inf], [0.0]])
    ids, top, lse = orc.top_logits(np.ones((2, 1)), W, 4, np.array([1]))
    assert ids[1].tolist() == [1, 3, 2, 0] and top[1].tolist() == [3.0, 3.0, 2.0, 1.0]
    assert abs(lse[1] - math.log(2 * math.exp(3) + math.exp(2) + math.exp(1) + 1)) < 1e-14
    assert ids[0].tolist() == [-1] * 4 and top[0].tolist() == [0.0] * 4 and lse[0] == 0.0
    ids, top, _ = orc.top_logits(np.ones((1, 1)), W, 6)
    assert ids[0].tolist() == [1, 3, 2, 0, 5, -1] and top[0, 5] == -np.inf


def test_masses_by_hand():
    ids = np.array([[0, 7, -1, 2], [9, -1, -1, 12], [1, 2, 3, 3]])
    l = np.array([[0.0, 5.0, 1.0, math.log(3.0)], [1.0, 2.0, 3.0, 4.0], [math.nan, -math.inf, 1.0, 1.0]])
    t = orc.teacher_masses(ids, l, None, 5)
    assert np.allclose(t, [[0.25, 0, 0, 0.75], [0, 0, 0, 0], [0, 0, 0.5, 0.5]], atol=1e-15)
    t = orc.teacher_masses(ids, l, np.log([8.0, 1.0, math.e * 4]), 5)
    assert np.allclose(t, [[0.125, 0, 0, 0.375], [0, 0, 0, 0], [0, 0, 0.25, 0.25]], atol=1e-15)


def test_cross_entropy_of_a_uniform_head_in_closed_form():
    rng = np.random.default_rng(1)
    H, V = rng.normal(size=(4, 3)), 8
    r = orc.cross_entropy(H, np.zeros((V, 3)), [2, -100, 5, 8], weight=np.array([2.0, 1.0, 1.0, 1.0]))
    assert np.allclose(r["row"], [-math.log(8), 0, -math.log(8), 0]) and abs(r["loss"] - 3 * math.log(8) / 4) < 1e-15
    want = np.zeros((V, 3))
    for i, y, w in ((0, 2, 2.0), (2, 5, 1.0)):
        want += np.outer((np.full(V, 1 / 8) - (np.arange(V) == y)) * w / 4, H[i])
    assert np.allclose(r["dW"], want, atol=1e-16) and not r["dH"].any()
    assert np.allclose(r["entropy"], [math.log(8), 0, math.log(8), 0])


def test_cross_entropy_agrees_with_torch():
    g = torch.Generator().manual_seed(5)
    H, W = torch.randn(9, 6, dtype=torch.float64, generator=g), torch.randn(11, 6, dtype=torch.float64, generator=g)
    y = torch.tensor([3, 0, -100, 10, 5, 5, 1, -100, 9])
    h, w = H.clone().requires_grad_(), W.clone().requires_grad_()
    loss = torch.nn.functional.cross_entropy(h @ w.T, y, reduction="sum") / 9
    loss.backward()
    r = orc.cross_entropy(H.numpy(), W.numpy(), y.numpy())
    assert abs(r["loss"] - float(loss.detach())) < 1e-14
    assert np.allclose(r["dH"], h.grad.numpy(), atol=1e-15) and np.allclose(r["dW"], w.grad.numpy(), atol=1e-15)


def test_distillation_on_the_whole_vocabulary_is_the_divergence_and_vanishes_at_the_teacher():
    rng = np.random.default_rng(2)
    H, W, Wt = rng.normal(size=(5, 4)), rng.normal(size=(6, 4)), rng.normal(size=(6, 4))
    ids, top, lse = orc.top_logits(H, Wt, 6)
    for tl in (None, lse):
        r = orc.distill(H, W, ids, top, tl)
        t = torch.softmax(torch.from_numpy(H @ Wt.T), 1)
        want = torch.nn.functional.kl_div(torch.log_softmax(torch.from_numpy(H @ W.T), 1), t, reduction="none").sum(1).numpy()
        assert np.allclose(r["row"], want, atol=1e-14) and abs(r["loss"] - want.mean()) < 1e-14 and np.allclose(r["mass"], 1)
        same = orc.distill(H, Wt, ids, top, tl)
        assert np.abs(same["row"]).max() < 1e-14 and np.abs(same["dH"]).max() < 1e-14 and np.abs(same["dW"]).max() < 1e-14


def test_one_place_renormalised_is_cross_entropy():
    rng = np.random.default_rng(3)
    H, W = rng.normal(size=(7, 4)), rng.normal(size=(9, 4))
    y, w = rng.integers(0, 9, 7), rng.normal(size=7)
    rows = np.array([0, 2, 3, 6])
    a = orc.distill(H, W, y[:, None], rng.normal(size=(7, 1)), None, rows, w, norm_rows=6)
    b = orc.cross_entropy(H, W, y, rows, w, norm_rows=6)
    assert np.allclose(a["row"], -b["row"]) and abs(a["loss"] - b["loss"]) < 1e-15 and np.allclose(a["dW"], b["dW"]) and np.allclose(a["dH"], b["dH"])


def test_a_token_in_two_places_counts_with_both():
    H, W = np.array([[1.0, 0.5]]), np.random.default_rng(4).normal(size=(5, 2))
    l = np.log(np.array([[0.2, 0.3, 0.5]]))
    a = orc.distill(H, W, np.array([[3, 1, 3]]), l)
    b = orc.distill(H, W, np.array([[3, 1]]), np.log(np.array([[0.7, 0.3]])))
    assert np.allclose(a["dz"], b["dz"], atol=1e-15)


@pytest.mark.parametrize("case", ["ce", "penalty", "renormalised", "tail"])
def test_gradients_match_finite_differences(case):
    rng = np.random.default_rng(7)
    n, d, V, k = 6, 4, 9, 3
    H, W, w = rng.normal(size=(n, d)), rng.normal(size=(V, d)), rng.normal(size=n)
    ids = np.stack([rng.permutation(V)[:k] for _ in range(n)])
    ids[1, 2], ids[4] = -1, -1
    l, lse, rows = rng.normal(size=(n, k)), 3 + rng.normal(size=n), np.array([0, 1, 3, 4, 5])

    def f(H, W):
        if case in ("ce", "penalty"):
            return orc.cross_entropy(H, W, ids[:, 0], rows, w, 0.3 if case == "penalty" else 0.0)
        return orc.distill(H, W, ids, l, None if case == "renormalised" else lse, rows, w)

    r, e = f(H, W), 1e-6
    for X, D in ((H, r["dH"]), (W, r["dW"])):
        for at in np.ndindex(X.shape):
            old = X[at]
            X[at] = old + e
            up = f(H, W)["loss"]
            X[at] = old - e
            down = f(H, W)["loss"]
            X[at] = old
            assert abs((up - down) / (2 * e) - D[at]) < 2e-9
    assert not r["dH"][[2, 4]].any()
