"""The forms of the gate's kernel, one by one, against the definition in 64 bits: choices exactly, weights within what fp32 rounds."""
import numpy as np
import pytest
import torch

import gate_cases as G
from oracle import front_oracle as F

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of fp32, relative


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def choose(moe, logits, bias, k, groups, kept, best, scores, renorm=True, scale=1.0, Es=0):
    T, E = logits.shape
    idx, w = torch.full((T + 1, k + Es), -7, dtype=torch.int32, device="cuda"), torch.full((T + 1, k + Es), -7.0, device="cuda")
    moe.moe_gate_fwd(moe.Shape(T, 64, 64, E, k, Es, renorm), moe.Gate(scores, groups, kept, best, scale), gpu(logits), gpu(bias), idx, w)
    torch.cuda.synchronize()
    assert (idx[T] == -7).all() and (w[T] == -7.0).all()   # rows behind the last
    return idx[:T].cpu().numpy(), w[:T].cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("T", [5, 5000])
@pytest.mark.parametrize("E,k,groups,kept", [(16, 4, 4, 2), (16, 2, 4, 1), (64, 8, 8, 3), (256, 8, 8, 4), (96, 6, 3, 1), (256, 12, 16, 5), (130, 20, 65, 30)])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_biases_whose_sums_leave_fp32(moe, scores, E, k, groups, kept, T):
    """A group's score is the sum of two c in 64 bits, also where it is past the largest number of 32; infinite biases are equal."""
    rng = np.random.default_rng([T, E])
    logits = rng.normal(size=(T, E)).astype(np.float32)
    for values in ([0.0, 2e38, 2.5e38, 3e38, 3.4e38], [0.0, 0.0, 1e38, 3e38, np.inf], [-2e38, -3e38, -9e29, 0.0, 3e38]):
        bias = rng.choice(np.array(values, np.float32), size=E)
        idx, w = choose(moe, logits, bias, k, groups, kept, 2, scores)
        some = np.unique(np.r_[0, T - 1, rng.integers(0, T, 60)])
        want, want_w = F.gate_fwd(logits[some], bias, k, scores, groups, kept, 2)
        assert np.array_equal(idx[some], want), values
        # exponentials of arguments up to 10 (their size times U, 2 U for the function), sums over k, two divisions
        assert (np.abs(w[some] - want_w) <= 60 * U * want_w).all()


def spread(logits):
    """How far apart the live logits of a row lie, at most: the exponentials' arguments (past 200 they are 0)."""
    l = np.where(logits > G.MASKED, logits, np.nan).astype(np.float64)
    l = l[~np.isnan(l).all(1)]
    return float(min((np.nanmax(l, 1) - np.nanmin(l, 1)).max(), 200.0)) if len(l) else 0.0


@pytest.mark.parametrize("form", G.FORMS, ids=lambda f: "-".join(map(str, f)))
def test_a_form_against_the_definition(moe, form):
    for n, case in enumerate(G.FORMS[form]):
        T, E, k, groups = case
        assert moe.gate_form(moe.Shape(T, 64, 64, E, k), moe.Gate("sigmoid", groups)) == form
        kept, best = G.groups_of(case)
        for scores in ("softmax", "sigmoid"):
            for mask in G.MASKS:
                for with_bias in (True, False):
                    print(case, scores, mask, with_bias, flush=True)
                    renorm = (n == 0) == (scores == "softmax")
                    logits, bias = G.make(case, mask, scores)
                    bias = bias if with_bias else None
                    idx, w = choose(moe, logits, bias, k, groups, kept, best, scores, renorm, 2.5, n)
                    args = gpu(logits), gpu(bias), k, scores, groups, kept, best
                    want, want_w, rating = G.gate_fwd(*args, renorm, 2.5)
                    want, want_w = want.cpu().numpy(), want_w.cpu().numpy()
                    other = np.nonzero((idx[:, :k] != want).any(1))[0]
                    for t in other:   # (of some masks, and only by the doubt about its groups)
                        left = G.choices_in_doubt(args[0][t:t + 1], *args[1:], rating[t:t + 1])
                        assert mask == "ties" and any(np.array_equal(c.cpu().numpy(), idx[t, :k]) for c in left), (case, scores, mask, with_bias, t)
                    assert len(other) <= T // 8, (case, scores, mask, with_bias, len(other))
                    assert (idx[:, k:] == np.arange(E, E + n)).all() and (w[:, k:] == 1).all()
                    # an exponential's argument is rounded and its factor too: 1.5 U of the argument's size; the function, the reciprocal, the sum of 32 and 6
                    # and the products are off by 1 or 2 U each
                    w, want_w, logits = (np.delete(v, other, 0) for v in (w, want_w, logits))
                    off = np.abs(w[:, :k] - want_w)
                    assert (off <= (2 * spread(logits) + 60) * U * want_w + 1e-37).all(), (case, scores, mask, with_bias, off.max())


@pytest.mark.parametrize("E,k", [(8, 6), (12, 5), (64, 40), (61, 9), (256, 20)])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_a_slot_without_weight_has_no_gradient_whatever_comes_in_there(moe, scores, E, k):
    """A token with fewer experts than choices: the masked ones' slots have weight 0, and what the experts' side says of these (NaN, an infinity) is not read."""
    T = 37
    rng = np.random.default_rng([T, E, k])
    logits = rng.normal(size=(T, E)).astype(np.float32)
    logits[rng.random((T, E)) < 0.8] = -np.inf
    logits[0], logits[1] = -np.inf, 1.0
    counts = rng.integers(0, 9, E).astype(np.int32)
    dw = gpu(rng.normal(size=(T, k)).astype(np.float32))
    for renorm in (True, False):
        s, gate = moe.Shape(T, 64, 64, E, k, 0, renorm), moe.Gate(scores, scale=2.5)
        idx, w = (gpu(v.astype(t)) for v, t in zip(choose(moe, logits, None, k, 1, 1, 1, scores, renorm, 2.5), (np.int32, np.float32)))
        none = w == 0
        assert none.any() and torch.equal(none, gpu(logits).gather(1, idx.long()) == -np.inf)
        for balance in (None, 0.5):
            got = []
            for value in (0.0, float("nan"), float("inf")):
                d = torch.empty(T, E, device="cuda")
                moe.moe_gate_bwd(s, gate, dw.masked_fill(none, value), gpu(logits), idx, w, None if balance is None else gpu(counts), balance or 0.0, d)
                got.append(d)
            assert torch.isfinite(got[0]).all() and torch.equal(got[0], got[1]) and torch.equal(got[0], got[2]), (renorm, balance)
            assert (got[0][gpu(logits) == -np.inf] == 0).all()
