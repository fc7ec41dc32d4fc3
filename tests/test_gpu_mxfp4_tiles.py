"""The grouped 4-bit products on large tiles: every height of an expert's last tile, contractions that end inside a stage or a batch of scales, with rows
of scales that are whole dwords and with others."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as M

pytestmark = pytest.mark.gpu

HEIGHTS = (1, 31, 32, 40, 64, 65, 96, 127, 130, 190, 193, 255, 256, 257, 300, 0, 480)


def _random(rng, *shape):
    """Codes of every kind, scales near each other; and the values."""
    q = rng.integers(0, 256, (*shape[:-1], shape[-1] // 2), dtype=np.uint8)
    s = rng.integers(122, 127, (*shape[:-1], shape[-1] // 32), dtype=np.uint8)
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), M.dequantize(q, s)


@pytest.mark.parametrize("k", [256, 288, 384, 512, 640, 1088, 1152, 2176, 4224])
def test_heights(moe, k):
    rng = np.random.default_rng(k)
    heights = HEIGHTS if k < 2000 else HEIGHTS[3::4]
    E, rows = len(heights), int(sum(heights))
    n = -(-16384 // rows) * 256 + 8   # (the last tile has 8 columns)
    offsets = np.concatenate([[0], np.cumsum(heights)]).astype(np.int32)
    xq, xs, x = _random(rng, rows, k)
    wq, ws, w = _random(rng, 1, n, k)
    wq, ws = wq.expand(E, -1, -1).contiguous(), ws.expand(E, -1, -1).contiguous()
    wq[-1] ^= 0x88   # (the last expert has the values of the others, negated)
    y = torch.full((rows + 1, n), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_gemm(xq, xs, torch.from_numpy(offsets).cuda(), wq, ws, y)
    want, far = M.grouped_gemm(x, w, np.array([0, rows]))
    want[offsets[-2]:] *= -1
    got = y.float().cpu().numpy().astype(np.float64)
    assert (got[rows] == 7.0).all()
    assert (np.abs(got[:rows] - want) <= far).all()


@pytest.mark.parametrize("d,f", [(256, 384), (320, 640), (1152, 256), (1088, 448)])
def test_pairs(moe, d, f):
    """The SwiGLU pair and the product after it, experts of every height."""
    rng = np.random.default_rng([d, f])
    heights = np.array([40, 1, 256, 0, 130, 70, 700, 199])
    heights = np.concatenate([heights, [max(0, -(-16384 * 128 // f) - heights.sum())]])
    E, rows = len(heights), int(heights.sum())
    offsets = np.concatenate([[0], np.cumsum(heights)]).astype(np.int32)
    x = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).bfloat16().cuda()
    parts = [_random(rng, E, f, d), _random(rng, E, f, d), _random(rng, E, d, f)]
    for q, s, _ in parts:
        s -= 3
    weights = [t for q, s, _ in parts for t in (q, s)]
    values = [M.dequantize(q.cpu().numpy(), s.cpu().numpy()) for q, s, _ in parts]
    shape = moe.Shape(rows, d, f, E, 1)
    wsp = torch.empty(moe.workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    y = torch.full((rows + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_ffn_fwd(shape, x, torch.from_numpy(offsets).cuda(), *weights, y[:rows], wsp)
    xv = x.float().cpu().numpy().astype(np.float64)
    for e in range(E):   # (of the many rows of the last expert the first and the last)
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        for a, b in ((lo, min(hi, lo + 300)), (max(lo, hi - 100), hi)):
            if a < b:
                want, far = M.grouped_ffn(xv[a:b], *[v[e:e + 1] for v in values], np.array([0, b - a]))
                assert (np.abs(y[a:b].float().cpu().numpy() - want) <= far).all(), (e, a, b)
    assert (y[rows] == 7.0).all()
