"""The layer for a few tokens where its launches change and at the ends of what its formats hold: gates of more than 16 experts made by the products' blocks,
slots past what they keep, scale codes at both ends, hidden values past bf16, gates far below zero."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx_oracle as M
from test_gpu_few import Case, _bf16, _f64

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])


def _bits(a):
    return W.f32_to_bf16_bits(np.asarray(a, np.float32))


@BOTH
@pytest.mark.parametrize("T,d,f,E,k,Es,renorm", [
    # router weights of at most 16 KB and more than 16 experts: groups of 16 in turn, the last one ragged
    (16, 64, 64, 128, 8, 0, 1),     # exactly 16 KB
    (9, 64, 128, 100, 6, 2, 1),
    (3, 128, 64, 33, 2, 1, 0),
    (1, 128, 128, 64, 3, 0, 1),     # exactly 16 KB, one token
    (16, 64, 64, 65, 5, 1, 0),      # past one logit per lane
    (16, 64, 64, 129, 8, 0, 1),     # a launch of its own again
])
def test_gates_made_by_every_block(moe, T, d, f, E, k, Es, renorm, mx):
    c = Case(T, d, f, E, k, Es, renorm, mx)
    buf = c.run(moe)
    idx, w = c.gate()
    assert np.array_equal(buf.topk_idx.cpu().numpy(), idx)
    assert np.allclose(buf.topk_w.cpu().numpy(), w, rtol=1e-5, atol=1e-8)
    c.check(buf, idx, w)


@BOTH
@pytest.mark.parametrize("T,E,k,Es", [(16, 60, 40, 0), (13, 300, 50, 2), (16, 257, 3, 0)])
def test_at_most_16_tokens_with_a_gate_launch(moe, T, E, k, Es, mx):
    """More than 512 slots, or more than 256 experts."""
    c = Case(T, 64, 128, E, k, Es, 1, mx)
    buf = c.run(moe)
    idx, w = c.gate()
    assert np.array_equal(buf.topk_idx.cpu().numpy(), idx)
    c.check(buf, idx, w)


@BOTH
def test_at_most_16_tokens_with_many_slots_of_one_expert(moe, mx):
    """... whose rows are more than an MFMA has, and more than a turn: the same expert several times for one token."""
    c = Case(16, 64, 128, 60, 40, 0, 1, mx)
    rng = np.random.default_rng(1)
    idx = np.where(rng.random((16, 40)) < 0.3, 7, rng.integers(0, 60, (16, 40))).astype(np.int32)
    assert (idx == 7).sum() > 64
    w = rng.random((16, 40)).astype(np.float32)
    want, far = np.zeros((16, 64)), np.zeros((16, 64))
    for j in range(40):
        y, b = M.layer_few(_f64(c.x), idx[:, j:j + 1], w[:, j:j + 1].astype(np.float64), *c.values)
        want += y
        far += b
    got = c.run(moe, (idx, w)).out.float().cpu().numpy()
    assert (np.abs(got - want) <= far + M.UBF16 * np.abs(want)).all()


@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("which", [0, 1, 2], ids=["gate", "up", "down"])
@pytest.mark.parametrize("low", [True, False], ids=["low", "high"])
def test_scale_codes_at_both_ends(moe, which, low, T):
    """Scale codes 0 .. 3 (2^-127 on) and 249 .. 252, in one of the three weights; the tokens and the other weights bring the products back into range."""
    c = Case(T, 128, 192, 3, 2, 0, 1, True)
    rng = np.random.default_rng([which, low])
    codes = (0, 4) if low else (249, 253)
    big = 100 if low else -100           # exponent that makes up for it
    q, s = [c.weights[2 * i] for i in range(3)], [c.weights[2 * i + 1] for i in range(3)]
    s[which].copy_(torch.from_numpy(rng.integers(*codes, tuple(s[which].shape)).astype(np.uint8)))
    if which < 2:
        c.x = _bits(W.bf16_bits_to_f32(c.x) * 2.0 ** big)
        s[1 - which].sub_(big) if big > 0 else s[1 - which].add_(-big)
        if which == 0:   # (G around 2^-24 or 2^24: H follows)
            s[2].add_(22) if low else s[2].sub_(22)
    else:
        s[1].add_(60) if low else s[1].sub_(60)
    c.values = [M.dequantize(a.cpu().numpy(), b.cpu().numpy()).transpose(0, 2, 1) for a, b in zip(q, s)]
    idx = np.stack([rng.permutation(3)[:2] for _ in range(T)]).astype(np.int32)
    w = rng.random((T, 2)).astype(np.float32)
    buf = c.run(moe, (idx, w))
    want, _ = M.layer_few(_f64(c.x), idx, w.astype(np.float64), *c.values)
    assert (np.abs(want) > 2.0 ** -120).any() and (np.abs(want) < 2.0 ** 120).all()
    c.check(buf, idx, w)


@BOTH
@pytest.mark.parametrize("T", [2, 20])
@pytest.mark.parametrize("g,u", [((2.0 ** 30, 2.0 ** 30), (2.0 ** 35, 2.0 ** 35)), ((2.0 ** 32 * 1.40625, 2.0 ** 32), (2.0 ** 31 * 1.421875, 2.0 ** 32))],
                         ids=["past fp32", "past bf16"])
def test_hidden_values_past_the_largest(moe, g, u, T, mx):
    """A hidden value that rounds to an infinity is one, and gives infinities of W_down's signs (no NaN).  g, u: a token's value and a weight."""
    d, f = 64, 64
    c = Case(T, d, f, 1, 1, 0, 1, mx)
    x = np.zeros((T, d))
    x[:, 0], x[:, 1] = g[0], u[0]
    c.x = _bits(x)
    wg, wu, wd = np.zeros((1, d, f)), np.zeros((1, d, f)), np.ones((1, f, d))
    wg[0, 0, 5], wu[0, 1, 5] = g[1], u[1]
    wd[0, 5, ::2] = -1.0
    if mx:
        c.weights = [torch.from_numpy(a).cuda() for v in (wg, wu, wd) for a in M.quantize(np.ascontiguousarray(v.transpose(0, 2, 1)))]
    else:
        c.weights = [_bf16(_bits(v)) for v in (wg, wu, wd)]
    out = c.run(moe, (np.zeros((T, 1), np.int32), np.ones((T, 1), np.float32))).out.float().cpu().numpy()
    want = np.where(np.arange(d) % 2 == 0, -np.inf, np.inf)
    assert np.array_equal(out, np.broadcast_to(want, out.shape)), out[0, :4]


@BOTH
@pytest.mark.parametrize("T", [16, 48])
def test_gates_far_below_zero(moe, T, mx):
    """G exact and down to -80, one hidden unit per output: out is silu(G) U to a bf16 rounding, relative to itself."""
    d = f = 64
    c = Case(T, d, f, 1, 1, 0, 1, mx)
    c.x = _bits(np.eye(d)[np.arange(T) % d])                       # token t takes row t of W_gate and W_up
    steps = np.array([0.5, 1, 1.5, 2, 3, 4, 6])
    rng = np.random.default_rng(2)
    wg = -steps[rng.integers(0, 7, (1, d, f))] * np.where(rng.random((1, 1, f)) < 0.5, 2.0, 8.0)   # (a column: a block, one scale) down to -48
    wg = np.where(np.arange(f) % 16 == 3, -64.0 - 16.0 * (np.arange(d) % 2)[None, :, None] * (0 if mx else 1), wg)
    wu, wd = np.ones((1, d, f)), np.eye(f)[None] * 1.0
    if mx:
        packed = [M.quantize(np.ascontiguousarray(v.transpose(0, 2, 1))) for v in (wg, wu, wd)]
        assert all(np.array_equal(M.dequantize(*p).transpose(0, 2, 1), v) for p, v in zip(packed, (wg, wu, wd)))
        c.weights = [torch.from_numpy(a).cuda() for p in packed for a in p]
    else:
        c.weights = [_bf16(_bits(v)) for v in (wg, wu, wd)]
    out = c.run(moe, (np.zeros((T, 1), np.int32), np.ones((T, 1), np.float32))).out.float().cpu().numpy().astype(np.float64)
    g = wg[0][np.arange(T) % d]
    want = g / (1 + np.exp(-g))
    # bf16 rounds by 2^-8 at most, H's remainder loses 2^-16, the exponential of a product rounded to fp32 |g| 2^-23 and a few units
    assert (np.abs(out - want) <= (2.0 ** -8 + 2.0 ** -16 + np.abs(g) * 2.0 ** -23 + 2.0 ** -20) * np.abs(want)).all()


@BOTH
def test_same_bits_whatever_turn_a_row_is_in(moe, mx):
    """Experts with more rows than a turn has: which of them share one follows no rule, and no sum depends on it."""
    c = Case(64, 256, 320, 2, 1, 1, 1, mx)
    first = c.run(moe).out
    for _ in range(20):
        assert torch.equal(c.run(moe).out, first)
