"""Microscaled 4-bit floating point: quantisation bit for bit, the grouped product and the FFN against the fp64 definition."""
import ctypes

import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx_oracle as M

pytestmark = pytest.mark.gpu


def _bf16(a):
    return torch.from_numpy(W.f32_to_bf16_bits(np.asarray(a, np.float32)).view(np.int16)).cuda().view(torch.bfloat16)


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _empty(*size):
    return torch.full(size, 0xA5, dtype=torch.uint8, device="cuda")


def _awkward(rng, rows, cols):
    """Values over the whole range of bf16: blocks of every magnitude, zeros, subnormals, ties, and a few that are not finite."""
    x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-130, 126, (rows, cols // 32)).repeat(32, 1)
    b = x.reshape(-1, 32)
    n = b.shape[0]
    b[rng.integers(0, n, max(1, n // 8))] = 0.0
    i = rng.integers(0, n, max(1, n // 4))   # multiples of a quarter of a power of two: ties of every code
    b[i] = rng.integers(-32, 33, (i.size, 32)) / 4.0 * 2.0 ** rng.integers(-100, 100, (i.size, 1))
    i = rng.integers(0, n, max(1, n // 8))
    b[i] = rng.integers(-8, 9, (i.size, 32)) * 2.0 ** -133   # the smallest bf16
    if n > 8:
        b[1, 3], b[3, 31], b[5, 0] = np.nan, np.inf, -np.inf
    return W.bf16_bits_to_f32(W.f32_to_bf16_bits(x.astype(np.float32))).astype(np.float64).reshape(rows, cols)


@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 64), (3, 96), (33, 1088), (257, 2048), (1003, 96), (2, 8192)])
def test_quantize_and_back_bit_for_bit(moe, rows, cols):
    rng = np.random.default_rng([rows, cols])
    x = _awkward(rng, rows, cols)
    q, s = _empty(rows, cols // 2), _empty(rows, cols // 32)
    moe.moe_mxfp4_quantize(_bf16(x), q, s)
    want_q, want_s = M.quantize(x)
    assert np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)
    back = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_dequantize(q, s, back)
    assert np.array_equal(_f64(back), M.dequantize(want_q, want_s), equal_nan=True)


@pytest.mark.parametrize("batch,rows,cols", [(1, 32, 8), (2, 64, 64), (3, 96, 136), (1, 1088, 72), (2, 288, 264), (5, 512, 128)])
def test_quantize_t_is_the_quantised_transpose(moe, batch, rows, cols):
    rng = np.random.default_rng([batch, rows, cols])
    w = np.stack([_awkward(rng, cols, rows).T for _ in range(batch)])
    q, s = _empty(batch, cols, rows // 2), _empty(batch, cols, rows // 32)
    moe.moe_mxfp4_quantize_t(_bf16(w), q, s)
    want_q, want_s = M.quantize(np.ascontiguousarray(w.transpose(0, 2, 1)))
    assert np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)


def test_every_code_at_every_scale_reads_back(moe):
    s = np.arange(256, dtype=np.uint8).reshape(256, 1)
    q = np.tile((np.arange(16) | (np.arange(16)[::-1] << 4)).astype(np.uint8), (256, 1))
    back = torch.empty(256, 32, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_dequantize(torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), back)
    want = M.dequantize(q, s)
    with np.errstate(over="ignore"):
        want = W.bf16_bits_to_f32(W.f32_to_bf16_bits(want.astype(np.float32)))   # (past the range: an infinity)
    got = back.float().cpu().numpy()
    assert np.array_equal(got[:255], want[:255]) and np.isnan(got[255]).all()


def _counts(rng, E, rows, dead=0):
    n = np.zeros(E, np.int64)
    alive = rng.permutation(E)[:E - dead]
    n[alive] = rng.multinomial(rows, np.full(alive.size, 1.0 / alive.size))
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def _mx(rng, *shape, std=1.0):
    """A quantised tensor on the device, and its values."""
    x = (rng.standard_normal(shape) * std * 2.0 ** rng.integers(-2, 3, (*shape[:-1], 1))).astype(np.float32)
    q, s = M.quantize(x.astype(np.float64))
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), M.dequantize(q, s)


@pytest.mark.parametrize("E,rows,n,k,dead", [
    (1, 1, 8, 32, 0), (1, 17, 64, 64, 0), (3, 1, 64, 128, 0), (4, 100, 72, 96, 1), (8, 300, 256, 512, 2), (5, 777, 328, 1088, 0), (130, 500, 64, 160, 60),
    (2, 1000, 512, 2048, 0), (1000, 64, 64, 64, 0), (7, 129, 1000, 224, 3), (2, 512, 640, 4128, 0),
    # enough rows for the large tiles: every height of an expert's last tile, results and contractions that end inside a tile
    (3, 9000, 520, 1088, 0), (40, 12000, 600, 288, 3), (2, 5000, 1024, 4128, 0), (300, 20000, 264, 256, 100), (9, 8300, 776, 672, 0),
])
def test_grouped_gemm(moe, E, rows, n, k, dead):
    rng = np.random.default_rng([E, rows, n, k])
    offsets = _counts(rng, E, rows, dead)
    xq, xs, x = _mx(rng, rows, k)
    wq, ws, w = _mx(rng, E, n, k, std=0.05)
    y = torch.full((rows + 1, n), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_gemm(xq, xs, torch.from_numpy(offsets).cuda(), wq, ws, y)
    want, far = M.grouped_gemm(x, w, offsets)
    got = _f64(y)
    assert (got[rows] == 7.0).all()
    assert (np.abs(got[:rows] - want) <= far).all()


def test_grouped_gemm_scales_and_nan_blocks(moe):
    """Scales far apart, a NaN block in one row of x and in one column of w."""
    rng = np.random.default_rng(5)
    xq, xs, _ = _mx(rng, 40, 256)
    wq, ws, _ = _mx(rng, 2, 64, 256)
    xs = (xs.to(torch.int32) + torch.from_numpy(rng.integers(-30, 30, tuple(xs.shape))).cuda()).to(torch.uint8)
    xs[3, 5], ws[1, 9, 2] = 255, 255
    offsets = np.array([0, 20, 40], np.int32)
    y = torch.empty(40, 64, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_gemm(xq, xs, torch.from_numpy(offsets).cuda(), wq, ws, y)
    x, w = M.dequantize(xq.cpu().numpy(), xs.cpu().numpy()), M.dequantize(wq.cpu().numpy(), ws.cpu().numpy())
    want, far = M.grouped_gemm(x, w, offsets)
    got = _f64(y)
    nan = np.isnan(want)
    assert nan.sum() == 64 + 20 and np.array_equal(np.isnan(got), nan)
    assert (np.abs(got - want)[~nan] <= far[~nan]).all()


@pytest.mark.parametrize("E,rows,d,f,dead", [
    (1, 1, 64, 64, 0), (4, 50, 128, 192, 1), (8, 512, 512, 1024, 0), (3, 333, 1088, 320, 0), (70, 256, 128, 64, 30), (2, 700, 320, 704, 0),
    (6, 7000, 320, 704, 1), (40, 9000, 576, 448, 4), (2, 5000, 1088, 512, 0),
])
def test_grouped_ffn(moe, E, rows, d, f, dead):
    rng = np.random.default_rng([E, rows, d, f])
    offsets = _counts(rng, E, rows, dead)
    x = W.bf16_bits_to_f32(W.f32_to_bf16_bits(rng.standard_normal((rows, d)).astype(np.float32))).astype(np.float64)
    gq, gs, wg = _mx(rng, E, f, d, std=1.5 / np.sqrt(d))
    uq, us, wu = _mx(rng, E, f, d, std=1.5 / np.sqrt(d))
    dq, ds, wd = _mx(rng, E, d, f, std=1.0 / np.sqrt(f))
    s = moe.Shape(rows, d, f, E, 1)
    ws = torch.empty(moe.workspace_bytes(s), dtype=torch.uint8, device="cuda")
    y = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_ffn_fwd(s, _bf16(x), torch.from_numpy(offsets).cuda(), gq, gs, uq, us, dq, ds, y, ws)
    want, far = M.grouped_ffn(x, wg, wu, wd, offsets)
    assert (np.abs(_f64(y) - want) <= far).all()


def test_offsets_past_32_bits(moe):
    """The last rows of a result of more than 2^32 bytes, from the last expert of weights of more than 2^32 values."""
    rng = np.random.default_rng(9)
    E, n, k, rows = 1024, 16384, 512, 150000
    wq, ws = torch.zeros(E, n, k // 2, dtype=torch.uint8, device="cuda"), torch.full((E, n, k // 32), 127, dtype=torch.uint8, device="cuda")
    xq, xs = torch.zeros(rows, k // 2, dtype=torch.uint8, device="cuda"), torch.full((rows, k // 32), 127, dtype=torch.uint8, device="cuda")
    tq, ts, x = _mx(rng, 5, k)
    vq, vs, w = _mx(rng, 1, n, k, std=0.05)
    xq[-5:], xs[-5:], wq[-1], ws[-1] = tq, ts, vq[0], vs[0]
    offsets = torch.full((E + 1,), rows - 5, dtype=torch.int32, device="cuda")
    offsets[0], offsets[E] = 0, rows
    y = torch.full((rows, n), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mxfp4_grouped_gemm(xq, xs, offsets, wq, ws, y)
    want, far = M.grouped_gemm(x, w, np.array([0, 5]))
    assert (np.abs(_f64(y[-5:]) - want) <= far).all()
    assert not y[:-5].any()


def test_products_on_another_stream_and_in_a_graph(moe):
    rng = np.random.default_rng(11)
    offsets = torch.from_numpy(_counts(rng, 4, 200, 1)).cuda()
    x = [_bf16(rng.standard_normal((200, 256))) for _ in range(3)]
    w = _mx(rng, 4, 192, 256)[:2] + _mx(rng, 4, 192, 256)[:2] + _mx(rng, 4, 256, 192)[:2]
    s = moe.Shape(200, 256, 192, 4, 1)
    ws = torch.empty(moe.workspace_bytes(s), dtype=torch.uint8, device="cuda")
    eager = []
    for v in x:
        y = torch.empty(200, 256, dtype=torch.bfloat16, device="cuda")
        moe.moe_mxfp4_grouped_ffn_fwd(s, v, offsets, *w, y, ws)
        eager.append(y)
    torch.cuda.synchronize()
    static, y = x[0].clone(), torch.empty(200, 256, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        moe.moe_mxfp4_grouped_ffn_fwd(s, static, offsets, *w, y, ws)
    torch.cuda.synchronize()
    assert torch.equal(y, eager[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_mxfp4_grouped_ffn_fwd(s, static, offsets, *w, y, ws)
    for v, want in list(zip(x, eager)) * 2:
        static.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_refusals(moe):
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8, device="cuda")  # noqa: E731
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    with pytest.raises(moe.MoeError):
        moe.moe_mxfp4_quantize(bf(4, 48), u8(4, 24), u8(4, 2))            # not whole blocks
    with pytest.raises(ValueError):
        moe.moe_mxfp4_quantize(bf(4, 64), u8(4, 31), u8(4, 2))            # too few codes
    with pytest.raises(ValueError):
        moe.moe_mxfp4_quantize(torch.zeros(4, 64, device="cuda"), u8(4, 32), u8(4, 2))
    with pytest.raises(ValueError):
        moe.moe_mxfp4_quantize(bf(64, 4).t(), u8(4, 32), u8(4, 2))        # not contiguous
    with pytest.raises(moe.MoeError):
        moe.moe_mxfp4_quantize_t(bf(1, 64, 12), u8(1, 12, 32), u8(1, 12, 2))
    with pytest.raises(ValueError):
        moe.moe_mxfp4_grouped_gemm(u8(4, 32), u8(4, 2), torch.zeros(3, dtype=torch.int32, device="cuda"), u8(2, 8, 16), u8(2, 8, 1), bf(4, 8))
    with pytest.raises(ValueError):   # offsets of another type
        moe.moe_mxfp4_grouped_gemm(u8(4, 32), u8(4, 2), torch.zeros(3, device="cuda"), u8(2, 8, 32), u8(2, 8, 2), bf(4, 8))


def test_nothing_to_do(moe):
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8, device="cuda")  # noqa: E731
    bf = lambda *n: torch.zeros(*n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    moe.moe_mxfp4_quantize(bf(0, 64), u8(0, 32), u8(0, 2))
    moe.moe_mxfp4_quantize_t(bf(0, 64, 64), u8(0, 64, 32), u8(0, 64, 2))
    moe.moe_mxfp4_dequantize(u8(0, 32), u8(0, 2), bf(0, 64))
    moe.moe_mxfp4_grouped_gemm(u8(0, 32), u8(0, 2), torch.zeros(3, dtype=torch.int32, device="cuda"), u8(2, 8, 32), u8(2, 8, 2), bf(0, 8))
    y = bf(4, 8)
    moe.moe_mxfp4_grouped_gemm(u8(4, 32), u8(4, 2), torch.zeros(3, dtype=torch.int32, device="cuda"), u8(2, 8, 32), u8(2, 8, 2), y)   # no expert has rows
    torch.cuda.synchronize()
