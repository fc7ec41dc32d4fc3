"""Pins of the fp64 definitions of routing and norm: closed forms, torch's operators, finite differences."""
import numpy as np
import pytest
import torch

from oracle import front_oracle as F
from oracle import moe_oracle as O


def _logits(T, E, seed=0):
    return np.random.default_rng(seed).normal(size=(T, E)).astype(np.float32)


def test_softmax_without_more_is_the_layers_own_gate():
    logits = _logits(37, 12)
    for renorm in (True, False):
        idx, w, _ = O.route_topk(logits, 3, 2, renorm)
        got = F.gate_fwd(logits, None, 3, "softmax", renorm=renorm, n_shared=2)
        assert np.array_equal(got[0], idx)
        np.testing.assert_allclose(got[1], w, rtol=1e-12)


def test_worked_example():
    # two groups of three; sigmoid scores 0.5 at 0; the bias moves the choice, not the weights
    logits = np.array([[0.0, 2.0, -1.0, 1.0, 1.5, 0.5]], np.float32)
    s = 1 / (1 + np.exp(-logits[0].astype(np.float64)))
    # best two: 0.881 + 0.5 = 1.381 against 0.818 + 0.731 = 1.549: the second group
    idx, w = F.gate_fwd(logits, None, 2, "sigmoid", groups=2, kept=1, best=2, renorm=True, scale=2.0)
    assert idx.tolist() == [[4, 3]]
    np.testing.assert_allclose(w[0], 2 * s[[4, 3]] / s[[4, 3]].sum())
    bias = np.array([0.3, 0, 0, 0, 0, 0], np.float32)   # 0.881 + 0.8: the first
    idx, w = F.gate_fwd(logits, bias, 2, "sigmoid", groups=2, kept=1, best=2, renorm=False)
    assert idx.tolist() == [[1, 0]]
    np.testing.assert_allclose(w[0], s[[1, 0]])


def test_masked_experts_come_last_and_ties_go_to_the_lowest():
    ninf = -np.inf
    logits = np.array([[ninf, 1, 1, np.nan, -1e30, 1], [ninf] * 6, [np.inf, 0, 0, 0, 0, -3e38]], np.float32)
    idx, w = F.gate_fwd(logits, None, 4, "softmax")
    assert idx.tolist() == [[1, 2, 5, 0], [0, 1, 2, 3], [0, 1, 2, 3]]
    np.testing.assert_allclose(w, [[1 / 3, 1 / 3, 1 / 3, 0], [0, 0, 0, 0], [1, 0, 0, 0]])
    idx, _ = F.gate_fwd(logits, None, 2, "sigmoid", groups=2, kept=1, best=2)
    assert idx.tolist() == [[1, 2], [0, 1], [0, 1]]


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("balance", [0.0, 3.0])
def test_gate_gradient_by_differences(scores, renorm, balance):
    T, E, k, scale = 4, 7, 3, 1.5
    rng = np.random.default_rng(3)
    logits = _logits(T, E, 4)
    idx, w = F.gate_fwd(logits, None, k, scores, renorm=renorm, scale=scale)
    dw = rng.normal(size=(T, k))
    counts = np.bincount(idx.reshape(-1), minlength=E)
    L = lambda l: float((F.gate_weights(l, idx, scores, renorm, scale) * dw).sum()) + F.balance_loss(l, counts, k, scores, balance)  # noqa: E731
    got, loss, size = F.gate_bwd(dw, logits, idx, w, k, scores, renorm, scale, counts, balance)
    assert abs(loss - F.balance_loss(logits, counts, k, scores, balance)) < 1e-12
    assert (np.abs(got) <= size + 1e-15).all()
    for t in range(T):
        for e in range(E):
            step = np.zeros((T, E))
            step[t, e] = 1e-5
            assert abs((L(logits + step) - L(logits - step)) / 2e-5 - got[t, e]) < 1e-8


def test_balance_loss_of_even_experts_is_balance():
    logits = np.zeros((10, 5), np.float32)
    for scores in ("softmax", "sigmoid"):
        assert abs(F.balance_loss(logits, np.full(5, 4), 2, scores, 0.7) - 0.7) < 1e-12


@pytest.mark.parametrize("centre", [True, False])
def test_norm_against_torch_and_its_gradient(centre):
    rng = np.random.default_rng(5)
    h, gamma, beta, dy = rng.normal(size=(5, 16)) + 0.5, rng.normal(size=16), rng.normal(size=16), rng.normal(size=(5, 16))
    ht, gt, bt = (torch.tensor(a, requires_grad=True) for a in (h, gamma, beta))
    y = (torch.nn.functional.layer_norm(ht, (16,), gt, bt, 1e-5) if centre else torch.nn.functional.rms_norm(ht, (16,), gt, 1e-5) + bt)
    got, mean, rstd = F.norm_fwd(h, gamma, beta, centre, 1e-5)
    np.testing.assert_allclose(got, y.detach().numpy(), rtol=1e-10, atol=1e-12)
    want = torch.autograd.grad(y, (ht, gt, bt), torch.tensor(dy))
    have = F.norm_bwd(dy, h, gamma, mean, rstd, centre)
    for a, b in zip(have, want):
        np.testing.assert_allclose(a, b.numpy(), rtol=1e-9, atol=1e-12)
    f = lambda a: float((F.norm_fwd(a, gamma, beta, centre, 1e-5)[0] * dy).sum())  # noqa: E731
    for at in ((0, 0), (2, 7), (4, 15)):
        step = np.zeros_like(h)
        step[at] = 1e-6
        assert abs((f(h + step) - f(h - step)) / 2e-6 - have[0][at]) < 1e-6
