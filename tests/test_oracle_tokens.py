"""Pins of the token-loss and embedding oracles: central differences, closed forms, torch's own float64 functions."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import elastic_oracle as orc
from oracle import token_oracle as tok


def _inputs(seed, M=7, V=11, vocab=9):
    rng = np.random.default_rng(seed)
    y = rng.normal(size=(M, V)) * 2
    t = rng.integers(0, vocab, M)
    w = rng.random(M) * (rng.random(M) < 0.8)
    return rng, y, t, w


def test_log_probs_against_torch():
    rng, y, t, w = _inputs(1)
    lp, p = tok.log_probs(y, t, 9, 0.7, np.ones(7, dtype=bool))
    want = torch.log_softmax(0.7 * torch.from_numpy(y[:, :9]), 1).numpy()
    np.testing.assert_allclose(lp, want[np.arange(7), t], rtol=1e-13)
    np.testing.assert_allclose(p, np.exp(want), rtol=1e-12)


@pytest.mark.parametrize("use_old,use_ref", [(True, True), (False, True), (True, False)])
def test_policy_gradient_against_differences(use_old, use_ref):
    rng, y, t, w = _inputs(2)
    adv = rng.normal(size=7)
    lp, _ = tok.log_probs(y, t, 9, 0.8, np.ones(7, dtype=bool))
    old0 = lp - np.array([0.5, -0.5, 0.05, 0.1, -0.1, 0.6, -0.6])
    ref = lp + 0.3 * rng.normal(size=7) if use_ref else None
    f = lambda v, old: tok.policy(v, t, w, adv, old, ref, 9, 0.8, 0.2, 0.3, 0.1 if use_ref else 0.0)  # noqa: E731
    # without `old` the ratio's reference is the current log probability: held fixed for the differences
    old = old0 if use_old else lp
    g = f(y, old0 if use_old else None)[2]
    num = np.zeros_like(y)
    for i in np.ndindex(*y.shape):
        h = np.zeros_like(y)
        h[i] = 1e-6
        num[i] = (f(y + h, old)[0][0] - f(y - h, old)[0][0]) / 2e-6
    np.testing.assert_allclose(g, num, atol=1e-8)


@pytest.mark.parametrize("kind,eps", [(0, 0.0), (0, 0.1), (1, 0.0), (2, 0.0)])
def test_preference_gradient_against_differences(kind, eps):
    rng, y, t, w = _inputs(3, M=12)
    begin = [1, 4, 6, 6, 10]                     # rows 0, 10, 11 belong to no sequence, one sequence is empty
    ref = rng.normal(size=4) - 5
    f = lambda v: tok.preference(v, t, w, begin, ref, 9, 1.1, kind, 0.2, eps)  # noqa: E731
    g = f(y)[2]
    num = np.zeros_like(y)
    for i in np.ndindex(*y.shape):
        h = np.zeros_like(y)
        h[i] = 1e-6
        num[i] = (f(y + h)[0][0] - f(y - h)[0][0]) / 2e-6
    np.testing.assert_allclose(g, num, atol=1e-8)
    assert not g[0].any() and not g[10:].any()


def test_pair_losses_against_torch():
    for x in (-30.0, -1.0, 0.0, 0.3, 25.0):
        v = torch.tensor(x, dtype=torch.float64, requires_grad=True)
        for kind, fn in ((0, lambda v: -0.9 * torch.nn.functional.logsigmoid(v) - 0.1 * torch.nn.functional.logsigmoid(-v)),
                         (1, lambda v: (v / 0.2 - 2.5) ** 2), (2, lambda v: torch.relu(1 - v))):
            v.grad = None
            want = fn(v)
            want.backward()
            got = tok.pair_loss(x, kind, 0.2, 0.1)
            np.testing.assert_allclose(got, (want.item(), v.grad.item()), rtol=1e-12, atol=1e-300)


def test_clip_factor():
    norm, f = tok.clip_factor([np.array([3.0]), np.array([4.0])], 2.5)
    assert norm == 5.0 and f == 0.5
    assert tok.clip_factor([np.array([3.0]), np.array([4.0])], 7.0) == (5.0, 1.0)
    assert tok.clip_factor([np.array([np.inf])], 1.0)[1] == 0.0


def test_embedding_gradient_against_differences():
    rng = np.random.default_rng(4)
    layers = [wl.embedding_layer(6, 8, 1.5), wl.Layer(8, 5, act=wl.ACT_GELU_TANH), wl.norm_layer(5)]
    W = [rng.normal(size=(6, 8)), rng.normal(size=(8, 5)), rng.normal(size=5)]
    b = [np.zeros(0), rng.normal(size=5), rng.normal(size=5)]
    ids = np.array([0, 3, 3, -1, 5, 6, 0, 3])                 # two ids outside the table, one row never used
    target = rng.normal(size=(8, 5))
    loss = lambda T: orc.mse_loss(orc.forward(layers, [T] + W[1:], b, ids).a[-1], target)  # noqa: E731
    saved = orc.forward(layers, W, b, ids)
    assert not saved.a[1][3].any() and not saved.a[1][5].any()
    _, dY = orc.mse_loss_grad(saved.a[-1], target)
    g, plan = orc.backward_masked(layers, W, saved, dY, np.array([1, 0, 0, 0, 0, 0]))
    num = np.zeros((6, 8))
    for i in np.ndindex(6, 8):
        h = np.zeros((6, 8))
        h[i] = 1e-6
        num[i] = (loss(W[0] + h) - loss(W[0] - h)) / 2e-6
    np.testing.assert_allclose(g[0], num, atol=1e-8)
    assert plan.deepest == 0 and not g[0][[1, 2, 4]].any()
