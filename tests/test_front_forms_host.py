"""The forms of the kernels in front of the experts: what is built is what some size reaches, no more and no less."""
import re

import numpy as np
import pytest
import torch

import gate_cases as G
import paper_2605_05049_amd as moe
from oracle import front_oracle as F
from test_kernel_resources import kernels  # noqa: F401


def _built(kernels, name):
    """Template arguments of a kernel's forms, from their mangled names."""
    found = (re.search(rf"\d{name}I((?:L[a-z]\d+E)+)E", k) for k in kernels)
    return {tuple(int(v) for v in re.findall(r"L[a-z](\d+)E", m.group(1))) for m in found if m}


def _lanes_of_chunks(cols):
    return next(lanes for lanes in (64, 128, 256, 512) if lanes == 512 or cols <= 24 * lanes)


def _chunks(cols, lanes):
    return -(-cols // (8 * lanes))


def test_forms_of_the_norm(kernels):  # noqa: F811
    """Lanes of a row and its chunks for every number of columns (the rules at the launches)."""
    fwd, bwd = set(), set()
    for cols in range(8, moe.NORM_COLS_MAX + 1, 8):
        few = 16 if cols <= 128 else 32 if cols <= 256 else None
        for lanes in (few or _lanes_of_chunks(cols), few or (128 if cols <= 512 else 256 if cols <= 2048 else 512)):   # without and with an addend
            fwd |= {(lanes, _chunks(cols, lanes), centre) for centre in (0, 1)}
        lanes = few or _lanes_of_chunks(cols)
        bwd |= {(lanes, _chunks(cols, lanes), centre, beta) for centre in (0, 1) for beta in (0, 1)}
    assert _built(kernels, "norm_fwd_kernel") == fwd and len(fwd) == 30
    assert _built(kernels, "norm_bwd_kernel") == bwd and len(bwd) == 48


def gate_forms():
    """form -> the cases (T, E, k, groups) that run it, over all E and groups, lists of every length and numbers of tokens on every side of the rule."""
    found = {}
    for E in range(1, 1025):
        for groups in (g for g in range(1, E + 1) if E % g == 0 and g <= 65):
            for k in (k for k in (1, 5, 9, 17) if k <= E):
                gate = moe.Gate("sigmoid", groups)
                for T in (1, 1500, 3000, 5000):
                    found.setdefault(moe.gate_form(moe.Shape(T, 64, 64, E, k), gate), []).append((T, E, k, groups))
    return found


def test_forms_of_the_gate(kernels):  # noqa: F811
    forms = gate_forms()
    assert _built(kernels, "gate_kernel") == {f for f in forms if f[0]}
    assert _built(kernels, "gate_general_kernel") == {f[2:3] for f in forms if not f[0]}


def test_form_refusals():
    import ctypes
    lib, s, g = moe.load_library(), ctypes.byref(moe.Shape(5, 64, 64, 8, 2)._c), ctypes.byref(moe.Gate()._c)
    form = (ctypes.c_int32 * 4)(*[7] * 4)
    assert lib.moe_gate_form(None, g, form) == -1 and lib.moe_gate_form(s, None, form) == -1 and lib.moe_gate_form(s, g, None) == -1
    assert lib.moe_gate_form(s, ctypes.byref(moe.Gate(groups=3)._c), form) == -2 and tuple(form) == (7, 7, 7, 7)
    assert moe.gate_form(moe.Shape(0, 64, 64, 8, 2), moe.Gate())[0] == 4 and moe.gate_form(moe.Shape(1 << 30, 64, 64, 8, 1), moe.Gate())[0] == 4


@pytest.mark.parametrize("form", G.FORMS, ids=lambda f: "-".join(map(str, f)))
def test_which_form_a_case_runs(form):
    """(The cases that are compared with the definition on the GPU: a changed rule shows here.)"""
    for T, E, k, groups in G.FORMS[form]:
        assert moe.gate_form(moe.Shape(T, 64, 64, E, k), moe.Gate("sigmoid", groups)) == form, (T, E, k, groups)
    assert form[0] == 0 or G.FORMS[form][1][2] == form[0]


def test_every_form_of_the_gate_has_its_cases():
    assert set(G.FORMS) == set(gate_forms())


@pytest.mark.parametrize("mask", G.MASKS)
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_the_definition_of_batches_is_that_of_tokens(scores, mask):
    for case in ((6, 16, 4, 4), (5, 60, 5, 6), (3, 130, 20, 65), (4, 96, 8, 1), (2, 6, 6, 2)):
        kept, best = G.groups_of(case)
        for with_bias in (True, False):
            for renorm in (True, False):
                logits, bias = G.make(case, mask, scores)
                bias = bias if with_bias else None
                want_idx, want = F.gate_fwd(logits, bias, case[2], scores, case[3], kept, best, renorm, 2.5)
                idx, w, _ = G.gate_fwd(torch.from_numpy(logits), None if bias is None else torch.from_numpy(bias), case[2], scores, case[3], kept, best, renorm, 2.5)
                assert np.array_equal(idx.numpy(), want_idx)
                np.testing.assert_allclose(w.numpy(), want, rtol=1e-12, atol=1e-300)


def test_choices_in_doubt():
    """Two groups whose scores are equal but for the order of adding: either stays, the third does not."""
    logits = torch.tensor([[0.5, 0.1, 0.5, 0.1, 0.4, 0.0]])
    bias = torch.tensor([0.25, 0.0, 0.0, 0.25, 0.0, 0.0])
    _, _, rating = G.gate_fwd(logits, bias, 2, "softmax", 3, 1, 2)
    assert abs(rating[0, 0] - rating[0, 1]) < G.DOUBT < rating[0, 0] - rating[0, 2]
    assert sorted(c.tolist() for c in G.choices_in_doubt(logits, bias, 2, "softmax", 3, 1, 2, rating)) == [[0, 1], [3, 2]]
    _, _, rating = G.gate_fwd(logits, None, 2, "softmax", 3, 2, 2)
    assert [c.tolist() for c in G.choices_in_doubt(logits, None, 2, "softmax", 3, 2, 2, rating)] == [[0, 2]]


def test_forms_of_the_gates_gradient(kernels):  # noqa: F811
    """Lanes of a token and chunks of 4 experts a lane, next to each other where E is a multiple of 4 (the rule at the launch)."""
    forms = set()
    for E in range(1, 1025):
        vec = E % 4 == 0
        lanes = 2 if vec and E <= 8 else 4 if vec and E <= 16 else 8
        while lanes < 64 and (16 if vec else 12) * lanes < E:
            lanes *= 2
        forms.add((lanes, -(-E // (4 * lanes)), int(vec)))
    assert _built(kernels, "gate_bwd_kernel") == forms
