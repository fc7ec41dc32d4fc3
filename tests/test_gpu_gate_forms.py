"""The forms of the gate's kernel, one by one, against the definition in 64 bits: choices exactly, weights within what fp32 rounds."""
import numpy as np
import pytest
import torch

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
