"""The grouped 4-bit products on every kernel at the ends of what the format holds: NaN blocks, scales far apart, rows that are not finite, gates far
below zero."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx_oracle as M

pytestmark = pytest.mark.gpu


def _random(rng, *shape, lo=100, hi=155):
    """Codes of every kind, scales far apart (2^-27 .. 2^27)."""
    q = rng.integers(0, 256, (*shape[:-1], shape[-1] // 2), dtype=np.uint8)
    s = rng.integers(lo, hi, (*shape[:-1], shape[-1] // 32), dtype=np.uint8)
    return q, s


# 64 large tiles of 256 x 256 at least: K a multiple of 128, any other K of 256 and more; and the small tiles
@pytest.mark.parametrize("rows,n,k", [(600, 8192, 256), (600, 8192, 1152), (600, 8192, 288), (600, 8192, 1088), (300, 64, 512), (300, 64, 96)])
def test_nan_blocks_and_scales_far_apart(moe, rows, n, k):
    rng = np.random.default_rng([rows, n, k])
    E, offsets = 3, np.array([0, 290 if rows == 600 else 40, rows - 130, rows], np.int32)
    xq, xs = _random(rng, rows, k)
    wq, ws = _random(rng, E, n, k)
    bad_rows, bad_columns = (3, offsets[1] - 1, offsets[1], rows - 1), ((0, 5), (1, n - 1), (2, n // 2 + 1))
    for i, r in enumerate(bad_rows):
        xs[r, (i * 5) % (k // 32)] = 255
    xs[bad_rows[0], -1] = 255   # the last block of a row
    for i, (e, c) in enumerate(bad_columns):
        ws[e, c, -1 if i == 1 else (i * 3) % (k // 32)] = 255
    y = torch.full((rows + 1, n), 7.0, dtype=torch.bfloat16, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    moe.moe_mxfp4_grouped_gemm(dev(xq), dev(xs), dev(offsets), dev(wq), dev(ws), y)
    got = y.float().cpu().numpy().astype(np.float64)
    assert (got[rows] == 7.0).all()
    x, w = M.dequantize(xq, xs), M.dequantize(wq, ws)
    want, far = M.grouped_gemm(x, w, offsets)
    nan = np.isnan(want)
    assert nan.sum() == 4 * n + sum(int(offsets[e + 1] - offsets[e]) - sum(offsets[e] <= r < offsets[e + 1] for r in bad_rows) for e, _ in bad_columns)
    assert np.array_equal(np.isnan(got[:rows]), nan)
    assert (np.abs(got[:rows] - want)[~nan] <= far[~nan]).all()


@pytest.mark.parametrize("scale", [0, 1, 127, 252, 254])
@pytest.mark.parametrize("rows,n,k", [(600, 8192, 256), (600, 8192, 288), (100, 64, 96)])
def test_scale_codes_at_both_ends(moe, rows, n, k, scale):
    """Every block of x at one scale code, and the weights' such that the products are around 1."""
    rng = np.random.default_rng([rows, k, scale])
    offsets = np.array([0, rows], np.int32)
    xq, xs = _random(rng, rows, k, lo=scale, hi=scale + 1)
    wq, ws = _random(rng, 1, n, k, lo=max(0, 254 - scale - 2), hi=min(254, 254 - scale + 3))
    y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    moe.moe_mxfp4_grouped_gemm(dev(xq), dev(xs), dev(offsets), dev(wq), dev(ws), y)
    want, far = M.grouped_gemm(M.dequantize(xq, xs), M.dequantize(wq, ws), offsets)
    assert (np.abs(y.float().cpu().numpy() - want) <= far).all()


@pytest.mark.parametrize("rows,d,f", [(50, 128, 192), (17000, 256, 1024), (17000, 320, 704)])
def test_rows_that_are_not_finite_stay_alone(moe, rows, d, f):
    """A NaN or an infinity in a row makes that whole row NaN and no other."""
    rng = np.random.default_rng([rows, d, f])
    E = 3
    offsets = torch.tensor([0, rows // 3, rows // 3, rows], dtype=torch.int32, device="cuda")
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    weights = [dev(a) for shape in ((E, f, d), (E, f, d), (E, d, f)) for a in _random(rng, *shape, lo=118, hi=123)]
    s = moe.Shape(rows, d, f, E, 1)
    ws = torch.empty(moe.workspace_bytes(s), dtype=torch.uint8, device="cuda")
    x = dev(rng.standard_normal((rows, d)).astype(np.float32)).bfloat16()
    clean, got = torch.empty_like(x), torch.empty_like(x)
    moe.moe_mxfp4_grouped_ffn_fwd(s, x, offsets, *weights, clean, ws)
    bad = (0, 7, rows // 3, rows - 1)
    for i, r in enumerate(bad):
        x[r, (37 * i) % d] = (float("nan"), float("inf"), -float("inf"))[i % 3]
    moe.moe_mxfp4_grouped_ffn_fwd(s, x, offsets, *weights, got, ws)
    nan = torch.zeros(rows, dtype=torch.bool, device="cuda")
    nan[list(bad)] = True
    assert got[nan].isnan().all() and torch.equal(got[~nan], clean[~nan]) and clean.isfinite().all()


@pytest.mark.parametrize("rows,d,f", [(64, 64, 64), (5000, 256, 1024), (5000, 320, 1024)])
def test_gates_far_below_zero(moe, rows, d, f):
    """G exact and down to -64, the same in a block of H: the codes of silu(G) U, relative to each block's own scale."""
    rng = np.random.default_rng([rows, d, f])
    steps = np.array([0.5, 1, 1.5, 2, 3, 4, 6])
    wg = -np.repeat(rng.choice(np.array([1, 2, 3, 4, 8, 16, 32, 48, 64.0]), (1, 1, f // 32)), 32, 2) * np.ones((1, d, 1))   # of a column one value
    wu = steps[rng.integers(0, 7, (1, d, f))]
    wd = np.zeros((1, f, d))
    wd[0, np.arange(min(d, f)), np.arange(min(d, f))] = 1.0       # output c is hidden unit c
    packed = [M.quantize(np.ascontiguousarray(v.transpose(0, 2, 1))) for v in (wg, wu, wd)]
    wg, wu, wd = (M.dequantize(*p).transpose(0, 2, 1) for p in packed)
    token = np.arange(rows) % d
    x = torch.eye(d, dtype=torch.bfloat16, device="cuda")[torch.from_numpy(token).cuda()].contiguous()
    s = moe.Shape(rows, d, f, 1, 1)
    ws = torch.empty(moe.workspace_bytes(s), dtype=torch.uint8, device="cuda")
    y = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    moe.moe_mxfp4_grouped_ffn_fwd(s, x, offsets, *[torch.from_numpy(a).cuda() for p in packed for a in p], y, ws)
    g, u = wg[0], wu[0]
    h = g / (1 + np.exp(-g)) * u
    # the exponential of a product rounded to fp32: |g| 2^-23, and a few units of fp32 for the rest
    hq, spread = M.quantized_spread(h, (np.abs(g) * 2.0 ** -23 + 2.0 ** -20) * np.abs(h))
    hq, spread = hq[:, :d], spread[:, :d]
    want = np.zeros((d, d))
    want[:, :min(d, f)], far = hq[:, :min(d, f)], np.zeros((d, d))
    far[:, :min(d, f)] = spread[:, :min(d, f)]
    assert (np.abs(y.float().cpu().numpy() - want[token]) <= far[token]).all()
