"""Residual sum, norm, router, gate and experts as they are used together: a training step of a block, and answering."""
import numpy as np
import pytest
import torch

from oracle import front_oracle as F
from paper_2605_05049_amd import serve

pytestmark = pytest.mark.gpu

T, D, FF, E, K, ES = 200, 256, 192, 16, 4, 1
GATES = {"sigmoid": ("sigmoid", 4, 2, 2, 2.5), "softmax": ("softmax", 8, 5, 1, 1.0), "plain": ("softmax", 1, 1, 1, 1.0)}


def normal(g, *s, std=1.0, mean=0.0):
    return (torch.randn(*s, generator=g) * std + mean).bfloat16().cuda()


def make(seed=0):
    g = torch.Generator().manual_seed(seed)
    n = E + ES
    return {"x": normal(g, T, D), "addend": normal(g, T, D, std=0.5), "gamma": normal(g, D, std=0.1, mean=1.0), "beta": normal(g, D, std=0.1),
            "w": (normal(g, n, D, FF, std=D ** -0.5), normal(g, n, D, FF, std=D ** -0.5), normal(g, n, FF, D, std=FF ** -0.5)),
            "w_router": normal(g, E, D, std=D ** -0.5), "bias": (0.02 * torch.randn(E, generator=g)).cuda(), "dout": normal(g, T, D), "dh": normal(g, T, D)}


def f64(t):
    return t.detach().double().cpu()


def definition(d, idx, gate, renorm, centre, balance):
    """The block in float64 with the kernels' choice of experts; (h, out, loss, leaves)."""
    scores, scale = gate[0], gate[4]
    leaf = {n: f64(d[n]).requires_grad_() for n in ("gamma", "beta", "w_router")}
    leaf["h"] = (d["x"].float() + d["addend"].float()).bfloat16().double().cpu().requires_grad_()
    for i, n in enumerate(("w_gate", "w_up", "w_down")):
        leaf[n] = f64(d["w"][i]).requires_grad_()
    h = leaf["h"]
    c = h - h.mean(1, keepdim=True) if centre else h
    y = c / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-6) * leaf["gamma"] + leaf["beta"]
    l = y @ leaf["w_router"].t()
    s = torch.sigmoid(l) if scores == "sigmoid" else torch.softmax(l, 1)
    w = s.gather(1, idx[:, :K])
    w = (w / w.sum(1, keepdim=True) if renorm else w) * scale
    loss = 0.0
    if balance:
        n = torch.bincount(idx[:, :K].reshape(-1), minlength=E).double()
        q = s / s.sum(1, keepdim=True)
        loss = balance * E / (K * T * T) * (q.sum(0) * n).sum()
    out = torch.zeros_like(y)
    ffn = lambda v, e: (torch.nn.functional.silu(v @ leaf["w_gate"][e]) * (v @ leaf["w_up"][e])) @ leaf["w_down"][e]  # noqa: E731
    for e in range(E):
        t, j = torch.nonzero(idx[:, :K] == e, as_tuple=True)
        if len(t):
            out = out.index_add(0, t, ffn(y[t], e) * w[t, j].unsqueeze(1))
    for e in range(E, E + ES):
        out = out + ffn(y, e)
    return h, out, loss, leaf


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("renorm", [1, 0])
@pytest.mark.parametrize("name", sorted(GATES))
def test_block_and_its_gradients(moe, name, renorm, centre):
    d, gate, balance = make(), GATES[name], 0.5 * T
    with_bias = name != "plain"
    buf = moe.MoeBlockBuffers(moe.Shape(T, D, FF, E, K, ES, renorm), centre)
    bias = d["bias"] if with_bias else None
    h, out = moe.block_forward(buf, d["x"], d["addend"], d["gamma"], d["beta"], *d["w"], d["w_router"], gate=moe.Gate(*gate), bias=bias)
    moe.block_backward(buf, h, d["dh"], d["dout"], d["gamma"], *d["w"], d["w_router"], gate=moe.Gate(*gate), balance=balance)
    torch.cuda.synchronize()
    L = buf.layer
    # the choice is the definition's for the kernels' own logits, the weights too
    idx, w = F.gate_fwd(L.logits.cpu().numpy(), None if bias is None else bias.cpu().numpy(), K, *gate[:4], bool(renorm), gate[4], ES)
    assert np.array_equal(idx, L.topk_idx.cpu().numpy())
    assert np.abs(w - L.topk_w.cpu().numpy()).max() <= 1e-5 * np.abs(w).max()
    h64, out64, loss, leaf = definition(d, L.topk_idx.cpu().long(), gate, renorm, centre, balance)
    assert torch.equal(h.cpu().double(), h64.detach())
    # the framework's bar, 2e-2 of the largest value: y, G, U, H, Y, dG, dU, dX are bf16 on the way
    near = lambda a, b, what: (f64(a) - b).abs().max() <= 2e-2 * b.abs().max() or pytest.fail(what)  # noqa: E731
    near(out, out64.detach(), "out")
    assert abs(L.balance_loss.item() - loss.item()) <= 1e-3 * loss.item()   # (the scores' own error, logits from a bf16 y)
    names = list(leaf)
    grads = dict(zip(names, torch.autograd.grad((out64 * f64(d["dout"])).sum() + loss + (h64 * f64(d["dh"])).sum(), [leaf[n] for n in names])))
    for n, got in (("h", buf.dh), ("gamma", buf.dgamma), ("beta", buf.dbeta), ("w_router", L.dw_router), ("w_gate", L.dw_gate), ("w_up", L.dw_up),
                   ("w_down", L.dw_down)):
        near(got, grads[n], n)
    # accumulating doubles the weights' gradients
    dgamma, dw = buf.dgamma.clone(), L.dw_router.clone()
    moe.block_backward(buf, h, d["dh"], d["dout"], d["gamma"], *d["w"], d["w_router"], accumulate=True, gate=moe.Gate(*gate), balance=balance)
    assert torch.allclose(buf.dgamma, 2 * dgamma, rtol=1e-5, atol=1e-5 * dgamma.abs().max().item())
    assert torch.allclose(L.dw_router, 2 * dw, rtol=1e-5, atol=1e-5 * dw.abs().max().item())


def test_layer_routed_by_a_gate_from_logits(moe):
    """The caller's logits in place of the router's: the same as the calls one by one."""
    d, g = make(1), moe.Gate(*GATES["sigmoid"])
    s = moe.Shape(T, D, FF, E, K, ES)
    logits = torch.randn(T, E, device="cuda")
    buf, two = moe.MoeLayerBuffers(s), moe.MoeLayerBuffers(s)
    moe.layer_forward(buf, d["x"], *d["w"], logits=logits, gate=g, bias=d["bias"])
    moe.layer_backward(buf, d["dout"], *d["w"], gate=g, logits=logits, balance=3.0)
    moe.moe_gate_fwd(s, g, logits, d["bias"], two.topk_idx, two.topk_w)
    moe.layer_forward(two, d["x"], *d["w"])
    moe.layer_backward(two, d["dout"], *d["w"], with_router=False)
    moe.moe_gate_bwd(s, g, two.dtopk_w, logits, two.topk_idx, two.topk_w, two.counts, 3.0, two.dlogits, two.balance_loss, two.ws)
    for n in ("topk_idx", "topk_w", "counts", "out", "dx", "dtopk_w", "dlogits", "balance_loss", "dw_gate", "dw_up", "dw_down"):
        assert torch.equal(getattr(buf, n), getattr(two, n)), n
    for bad in (dict(bias=d["bias"]), dict(gate=g)):
        with pytest.raises(ValueError):
            moe.layer_forward(buf, d["x"], *d["w"], **bad)
    with pytest.raises(ValueError):
        moe.layer_backward(buf, d["dout"], *d["w"], balance=1.0)


def test_captured_steps(moe):
    """A layer step with a gate by CapturedLayerStep, and a whole block in a graph: replays with other inputs, eager work between them."""
    d, g = make(2), moe.Gate(*GATES["sigmoid"])
    s = moe.Shape(T, D, FF, E, K, ES)
    captured, eager = moe.MoeLayerBuffers(s), moe.MoeLayerBuffers(s)
    step = moe.CapturedLayerStep(captured, d["x"], d["dout"], *d["w"], w_router=d["w_router"], gate=g, bias=d["bias"], balance=2.0)
    block, other = moe.MoeBlockBuffers(s, True), moe.MoeBlockBuffers(s, True)

    def run(b):
        h, out = moe.block_forward(b, d["x"], d["addend"], d["gamma"], d["beta"], *d["w"], d["w_router"], gate=g, bias=d["bias"])
        moe.block_backward(b, h, d["dh"], d["dout"], d["gamma"], *d["w"], d["w_router"], gate=g, balance=2.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(block)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(block)
    for seed in (3, 4, 5):
        new = make(seed)
        for n in ("x", "addend", "gamma", "beta", "w_router", "bias", "dout", "dh"):
            d[n].copy_(new[n])
        step.replay()
        moe.layer_forward(eager, d["x"], *d["w"], w_router=d["w_router"], gate=g, bias=d["bias"])
        moe.layer_backward(eager, d["dout"], *d["w"], x=d["x"], w_router=d["w_router"], gate=g, balance=2.0)
        torch.cuda.synchronize()
        for n in ("topk_idx", "topk_w", "out", "dx", "dlogits", "balance_loss", "dw_router", "dw_gate", "dw_up", "dw_down"):
            assert torch.equal(getattr(captured, n), getattr(eager, n)), n
        run(other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("h", "y", "mean", "rstd", "dh", "dgamma", "dbeta"):
            assert torch.equal(getattr(block, n), getattr(other, n)), n
        for n in ("out", "dx", "balance_loss", "dw_router"):
            assert torch.equal(getattr(block.layer, n), getattr(other.layer, n)), n


@pytest.mark.parametrize("mxfp4", [True, False])
def test_answering_through_a_gate_and_a_norm(moe, mxfp4):
    """Prompts and steps are what the entry points give, on the current stream, on another one, and captured."""
    d, g = make(6), moe.Gate(*GATES["sigmoid"])
    layer = serve.ServedLayer(d["w_router"], *d["w"], K, ES, mxfp4=mxfp4, gate=g, bias=d["bias"], norm=(d["gamma"], d["beta"], True, 1e-6))
    weights = moe.quantize_experts(*d["w"]) if mxfp4 else d["w"]
    for n in (1, 7, 64, T):
        x, a = d["x"][:n].contiguous(), d["addend"][:n].contiguous()
        h, y = torch.empty_like(x), torch.empty_like(x)
        moe.moe_norm_fwd(True, 1e-6, x, a, d["gamma"], d["beta"], h, y, None, None)
        s = moe.Shape(n, D, FF, E, K, ES)
        full = moe.MoeLayerBuffers(s, with_backward=False)
        logits, idx, w = torch.empty(n, E, device="cuda"), torch.empty(n, K + ES, dtype=torch.int32, device="cuda"), torch.empty(n, K + ES, device="cuda")
        moe.moe_router_gate_fwd(s, g, y, d["w_router"], d["bias"], logits, idx, w, full.ws)
        if n <= moe.FEW_TOKENS_MAX:
            few = moe.FewTokenBuffers(s)
            few.topk_idx.copy_(idx), few.topk_w.copy_(w)
            want = moe.layer_few_forward(few, y, weights)
        else:
            full.topk_idx.copy_(idx), full.topk_w.copy_(w)
            want = moe.layer_mxfp4_forward(full, y, weights) if mxfp4 else moe.layer_forward(full, y, *weights)
        got_h, got = layer.block(x, a)
        assert torch.equal(got_h, h) and torch.equal(got, want)
        assert torch.equal(layer(y), want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got_h, got = layer.block(x, a, stream=side)
        side.synchronize()
        assert torch.equal(got_h, h) and torch.equal(got, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got_h, got = layer.block(x, a)
        for _ in range(3):
            got_h.zero_(), got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got_h, h) and torch.equal(got, want)
            layer(y)
        h2, first = layer.block(x)
        assert h2 is x
    first, rows = serve.answer(layer, d["x"], 3, 2)
    assert first.shape == (T, D) and rows.shape == (2, 3, D) and torch.isfinite(rows.float()).all()
    with pytest.raises(ValueError):
        layer.block(d["x"], d["addend"][:5])
    with pytest.raises(ValueError):
        serve.ServedLayer(d["w_router"], *d["w"], K, ES, mxfp4=False).block(d["x"])


def test_bias_steps_even_the_loads(moe):
    d, g = make(7), moe.Gate("sigmoid")
    d["w_router"][:3] *= 3   # some experts are liked by many tokens
    layer = serve.ServedLayer(d["w_router"], *d["w"], K, ES, mxfp4=False, gate=g, bias=torch.zeros(E, device="cuda"))
    before, after = serve.balance(layer, d["x"], 200, 0.002)
    assert after < before


def test_command(moe, capsys):
    assert serve.main("--dims 256x192 --experts 8 --top-k 2 --shared 1 --prompt 80 --batch 2 --steps 3 --scores sigmoid --groups 4 --groups-kept 2 "
                      "--group-best 2 --scale 2.5 --norm layer --balance-steps 5".split()) == 0
    out = capsys.readouterr().out
    assert '"step_us"' in out and '"load_after"' in out
