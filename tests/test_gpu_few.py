"""The whole layer for a few tokens against the fp64 definition, on bf16 and on 4-bit weights."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import moe_oracle as O
from oracle import mx_oracle as M

pytestmark = pytest.mark.gpu


def _bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def _f64(bits):
    return W.bf16_bits_to_f32(bits).astype(np.float64)


class Case:
    def __init__(self, T, d, f, E, k, Es=0, renorm=1, mx=False, seed=0):
        sh = W.MoEShape(T, d, f, E, k, Es, renorm)
        self.sh = sh
        rng = np.random.default_rng([T, d, f, E, k, Es, seed])
        self.x = W.make_tokens(sh, seed)
        self.w_router = W.f32_to_bf16_bits((rng.standard_normal((E, d)) * (2.0 / np.sqrt(d))).astype(np.float32))
        std = (1.5 / np.sqrt(d), 1.5 / np.sqrt(d), 1.0 / np.sqrt(f))
        shapes = ((sh.E_total, d, f), (sh.E_total, d, f), (sh.E_total, f, d))
        bits = [W.f32_to_bf16_bits((rng.standard_normal(s) * v).astype(np.float32)) for s, v in zip(shapes, std)]
        if mx:
            packed = [M.quantize(np.ascontiguousarray(_f64(b).transpose(0, 2, 1))) for b in bits]
            self.values = [M.dequantize(*p).transpose(0, 2, 1) for p in packed]
            self.weights = [torch.from_numpy(a).cuda() for p in packed for a in p]
        else:
            self.values = [_f64(b) for b in bits]
            self.weights = [_bf16(b) for b in bits]

    def gate(self):
        logits = _f64(self.x) @ _f64(self.w_router).T
        return O.route_topk(logits.astype(np.float32), self.sh.k, self.sh.E_shared, bool(self.sh.renorm))[:2]

    def run(self, moe, routed=None, stream=None):
        s = moe.Shape.of(self.sh)
        buf = moe.FewTokenBuffers(s)
        buf.ws.fill_(0xA5)
        buf.out.fill_(9.0)
        if routed is not None:
            buf.topk_idx.copy_(torch.from_numpy(routed[0].astype(np.int32)))
            buf.topk_w.copy_(torch.from_numpy(routed[1].astype(np.float32)))
        moe.layer_few_forward(buf, _bf16(self.x), self.weights, w_router=None if routed is not None else _bf16(self.w_router), stream=stream)
        torch.cuda.synchronize()
        return buf

    def check(self, buf, idx, w):
        want, far = M.layer_few(_f64(self.x), idx, w.astype(np.float64), *self.values)
        got = buf.out.float().cpu().numpy().astype(np.float64)
        assert (np.abs(got - want) <= far).all(), float((np.abs(got - want) / far).max())


SHAPES = [
    # T, d, f, E, k, shared, renorm
    (1, 64, 64, 1, 1, 0, 1),
    (1, 512, 1024, 8, 2, 0, 1),
    (2, 64, 192, 3, 3, 1, 0),
    (3, 128, 320, 5, 2, 1, 1),
    (7, 320, 64, 66, 6, 2, 1),
    (16, 256, 448, 8, 2, 0, 0),
    (17, 192, 576, 9, 3, 2, 1),
    (31, 1088, 128, 13, 3, 1, 0),
    (33, 128, 1984, 2, 1, 0, 1),
    (48, 64, 64, 300, 8, 0, 1),
    (64, 128, 256, 4, 4, 0, 1),      # every expert has all tokens
    (64, 448, 192, 1024, 2, 0, 1),
    (63, 192, 128, 16, 2, 2, 1),
    (1, 4096, 64, 2, 1, 0, 1),
    (5, 64, 2048, 257, 1, 1, 1),
]


@pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])
@pytest.mark.parametrize("T,d,f,E,k,Es,renorm", SHAPES)
def test_layer_few(moe, T, d, f, E, k, Es, renorm, mx):
    if E + Es > 1024:
        pytest.skip("more experts than a layer has")
    c = Case(T, d, f, E, k, Es, renorm, mx)
    buf = c.run(moe)
    idx, w = c.gate()
    assert np.array_equal(buf.topk_idx.cpu().numpy(), idx)
    assert np.allclose(buf.topk_w.cpu().numpy(), w, rtol=1e-5, atol=1e-8)
    c.check(buf, idx, w)


@pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])
def test_rows_that_arrive_routed(moe, mx):
    """No router: ids and weights are given, one expert per row and skewed; and the same expert several times for one row."""
    c = Case(61, 128, 192, 7, 1, 0, 1, mx)
    rng = np.random.default_rng(3)
    idx = np.minimum(rng.geometric(0.5, (61, 1)) - 1, 6).astype(np.int32)
    w = rng.random((61, 1)).astype(np.float32)
    c.check(c.run(moe, (idx, w)), idx, w)
    c = Case(64, 64, 128, 3, 3, 1, 1, mx)
    idx = np.zeros((64, 4), np.int32)   # 256 rows of one expert
    idx[5] = 2
    w = rng.standard_normal((64, 4)).astype(np.float32)
    want = np.zeros((64, 64))
    far = np.zeros((64, 64))
    for j in range(4):   # (absolute values: the bound of a negative gate weight)
        y, b = M.layer_few(_f64(c.x), idx[:, j:j + 1], np.ones((64, 1)), *c.values)
        want += w[:, j:j + 1] * y
        far += np.abs(w[:, j:j + 1]) * b
    got = c.run(moe, (idx, w)).out.float().cpu().numpy()
    assert (np.abs(got - want) <= far + M.UBF16 * np.abs(want)).all()


@pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])
def test_a_token_that_is_not_finite_stays_alone(moe, mx):
    c = Case(20, 128, 192, 6, 2, 1, 1, mx)
    clean = c.run(moe).out.clone()
    x = c.x.copy()
    x[3, 17] = 0x7FC0
    x[11, 64] = 0x7F80
    bad = Case(20, 128, 192, 6, 2, 1, 1, mx)
    bad.x = x
    out = bad.run(moe).out
    keep = [t for t in range(20) if t not in (3, 11)]
    assert torch.equal(out[keep], clean[keep])
    assert out[3].isnan().all() and not out[11].isfinite().any()


def test_nan_blocks_of_weights(moe):
    c = Case(4, 128, 128, 2, 2, 0, 1, True)
    c.weights[5][1, 70, 2] = 255   # W_down, expert 1, output column 70
    out = c.run(moe).out
    nan = out.isnan()
    assert nan[:, 70].all() and nan.sum() == 4


def test_same_bits_every_time_and_on_another_stream(moe):
    for mx in (False, True):
        c = Case(29, 256, 320, 12, 3, 1, 1, mx)
        first = c.run(moe).out
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        for stream in (None, side, None):
            assert torch.equal(c.run(moe, stream=stream).out, first)


@pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])
def test_replayed_graph(moe, mx):
    cases = [Case(9, 256, 320, 12, 3, 1, 1, mx, seed=i) for i in range(3)]
    xs = [_bf16(c.x) for c in cases]
    s, w, wr = moe.Shape.of(cases[0].sh), cases[0].weights, _bf16(cases[0].w_router)
    buf = moe.FewTokenBuffers(s)
    eager = [moe.layer_few_forward(buf, x, w, w_router=wr).clone() for x in xs]
    static = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.layer_few_forward(buf, static, w, w_router=wr)
    for x, want in list(zip(xs, eager)) * 2:
        static.copy_(x)
        buf.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(buf.out, want)


def test_weights_past_32_bits(moe):
    """The last of experts whose weights take more than 2^32 bytes."""
    E, d, f = 72, 2048, 16384
    c = Case(2, d, f, 1, 1)
    w = []
    for v in c.weights:
        t = torch.empty(E, *v.shape[1:], dtype=torch.bfloat16, device="cuda")
        t[E - 1] = v[0]
        w.append(t)
    assert w[0].numel() * 2 > 2 ** 32
    buf = moe.FewTokenBuffers(moe.Shape(2, d, f, E, 1))
    buf.topk_idx.fill_(E - 1)
    buf.topk_w.copy_(torch.tensor([[1.0], [0.25]]))
    moe.layer_few_forward(buf, _bf16(c.x), w)
    want, far = M.layer_few(_f64(c.x), np.zeros((2, 1), np.int64), np.array([[1.0], [0.25]]), *c.values)
    assert (np.abs(buf.out.float().cpu().numpy() - want) <= far).all()


def test_as_the_layer_does(moe):
    """The same layer, both ways: within what bf16 storage of the intermediates costs the other one."""
    c = Case(24, 512, 1024, 8, 2, 1)
    out = c.run(moe).out.float()
    buf = moe.MoeLayerBuffers(moe.Shape.of(c.sh), with_backward=False)
    other = moe.layer_forward(buf, _bf16(c.x), *c.weights, w_router=_bf16(c.w_router)).float()
    assert ((out - other).abs().max() / other.abs().max()).item() <= 2e-2
    assert torch.equal(buf.topk_idx, c.run(moe).topk_idx)


def test_no_tokens(moe):
    s = moe.Shape(0, 64, 64, 4, 2)
    e = lambda *n, dtype=torch.bfloat16: torch.empty(*n, dtype=dtype, device="cuda")  # noqa: E731
    moe.moe_layer_few_fwd(s, e(0, 64), e(4, 64), e(4, 64, 64), e(4, 64, 64), e(4, 64, 64), e(0, 64), e(0, 2, dtype=torch.int32),
                          e(0, 2, dtype=torch.float32), e(1, dtype=torch.uint8))


def test_refusals(moe):
    with pytest.raises(ValueError):
        moe.FewTokenBuffers(moe.Shape(65, 64, 64, 4, 2))
    with pytest.raises(ValueError):
        moe.FewTokenBuffers(moe.Shape(64, 64, 64, 128, 65))   # 4160 slots
    c = Case(4, 64, 64, 4, 2)
    buf = moe.FewTokenBuffers(moe.Shape.of(c.sh))
    with pytest.raises(moe.MoeError):
        moe.moe_layer_few_fwd(buf.shape, _bf16(c.x), _bf16(c.w_router), *c.weights, buf.out, buf.topk_idx, buf.topk_w, buf.ws[:256])
    with pytest.raises(ValueError):
        moe.moe_layer_few_fwd(buf.shape, _bf16(c.x), _bf16(c.w_router), c.weights[0][:2].contiguous(), *c.weights[1:], buf.out, buf.topk_idx,
                              buf.topk_w, buf.ws)
