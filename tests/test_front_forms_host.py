"""The forms of the kernels in front of the experts: what is built is what some size reaches, no more and no less."""
import re

import paper_2605_05049_amd as moe
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
