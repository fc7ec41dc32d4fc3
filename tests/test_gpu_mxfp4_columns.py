"""The grouped 4-bit products on large tiles that their columns do not fill."""
import numpy as np
import pytest
import torch

import paper_2605_05049_amd
from oracle import mx_oracle as M
from test_gpu_mxfp4_tiles import _random

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n,k", [(45000, 96, 512), (45000, 96, 544), (35000, 120, 640), (22000, 192, 1152), (22000, 200, 736), (17000, 248, 1024),
                                      (9000, 504, 672), (66000, 192, 256), (66000, 192, 320)])
def test_product(moe, rows, n, k):
    assert paper_2605_05049_amd.mxfp4_grouped_gemm_large_tiles(4, rows, n, k)
    rng = np.random.default_rng([rows, n, k])
    offsets = np.array([0, 700, 700, 1013, rows], np.int32)
    xq, xs, x = _random(rng, rows, k)
    wq, ws, w = _random(rng, 4, n, k)
    y = torch.full((rows + 1, n), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_gemm(xq, xs, torch.from_numpy(offsets).cuda(), wq, ws, y)
    got = y.float().cpu().numpy().astype(np.float64)
    assert (got[rows] == 7.0).all()
    for lo, hi in ((0, 1500), (rows - 700, rows)):   # (of the last expert's rows the first and the last)
        want, far = M.grouped_gemm(x[lo:hi], w, np.clip(offsets, lo, hi) - lo)
        assert (np.abs(got[lo:hi] - want) <= far).all()


@pytest.mark.parametrize("rows,d,f", [(33000, 512, 64), (33000, 576, 64), (11500, 1024, 192), (17000, 512, 128)])
def test_ffn(moe, rows, d, f):
    rng = np.random.default_rng([rows, d, f])
    offsets = np.array([0, 300, 300, 533, rows], np.int32)
    parts = [_random(rng, 4, f, d), _random(rng, 4, f, d), _random(rng, 4, d, f)]
    for q, s, _ in parts:
        s -= 3
    values = [M.dequantize(q.cpu().numpy(), s.cpu().numpy()) for q, s, _ in parts]
    x = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).bfloat16().cuda()
    shape = moe.Shape(rows, d, f, 4, 1)
    wsp = torch.empty(moe.mxfp4_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_ffn_fwd(shape, x, torch.from_numpy(offsets).cuda(), *[t for q, s, _ in parts for t in (q, s)], y[:rows], wsp)
    assert (y[rows] == 7.0).all()
    xv, got = x.float().cpu().numpy().astype(np.float64), y.float().cpu().numpy().astype(np.float64)
    for lo, hi in ((0, 900), (rows - 300, rows)):
        want, far = M.grouped_ffn(xv[lo:hi], *values, np.clip(offsets, lo, hi) - lo)
        assert (np.abs(got[lo:hi] - want) <= far).all()
