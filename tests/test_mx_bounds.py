"""The bound of silu in fp32 that the tests of the 4-bit FFN and of the layer for a few tokens take, against an emulation in which every step rounds."""
import numpy as np
import pytest

from oracle import mx_oracle as M


def _silu(g, exp2_off, reciprocal_off):
    """silu(g) = g / (1 + 2^t), t = -g log2 e, each step in fp32; 2^t and the reciprocal within a unit in the last place: half of one from these, half from
    the rounding."""
    f = np.float32
    t = (-g * f(np.log2(np.e))).astype(f)
    e = (np.exp2(t.astype(np.float64)) * (1 + exp2_off * M.U32)).astype(f)
    s = (f(1) + e).astype(f)
    r = (1 / s.astype(np.float64) * (1 + reciprocal_off * M.U32)).astype(f)
    return (g * r).astype(f)


@pytest.mark.parametrize("lo,hi", [(0, 2), (2, 80), (-2, 0), (-5, -2), (-10, -5), (-20, -10), (-40, -20), (-80, -40)])
def test_silu_error(lo, hi):
    g = np.random.default_rng(abs(hi)).uniform(lo, hi, 200000).astype(np.float32)
    G = g.astype(np.float64)
    want = G / (1 + np.exp(-G))
    for a in (-1, 0, 1):
        for b in (-1, 0, 1):
            off = np.abs(_silu(g, a, b) - want) / np.maximum(np.abs(want), 1e-300)
            assert (off <= M.silu_error(G)).all()
            assert (off <= (6 + 1.25 * np.maximum(-G, 0)) * M.U32).all()   # (what the kernel's comment says)
    if hi <= -10:   # a constant does not hold here
        assert off.max() > M.EXP
