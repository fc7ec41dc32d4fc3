"""The operators that answer, together: quantised once, a prompt through the grouped products, then step by step."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from oracle import mx_oracle as M
from paper_2605_05049_amd import serve

pytestmark = pytest.mark.gpu

E, K, ES, D, F = 8, 2, 1, 256, 448


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.fixture(scope="module")
def model():
    g = torch.Generator().manual_seed(11)
    normal = lambda *s, std: (torch.randn(*s, generator=g) * std).bfloat16().cuda()  # noqa: E731
    weights = [normal(E + ES, D, F, std=D ** -0.5), normal(E + ES, D, F, std=D ** -0.5), normal(E + ES, F, D, std=F ** -0.5)]
    return normal(E, D, std=2 * D ** -0.5), weights, normal(100, D, std=1.0)


@pytest.mark.parametrize("batch", [1, 5, 20, 64])
def test_steps_follow_the_definition(moe, model, batch):
    w_router, weights, x = model
    layer = serve.ServedLayer(w_router, *weights, K, ES)
    values = [M.dequantize(layer.weights[2 * i].cpu().numpy(), layer.weights[2 * i + 1].cpu().numpy()).transpose(0, 2, 1) for i in range(3)]
    first, rows = serve.answer(layer, x, batch, 3)
    assert first.shape == (100, D) and isinstance(layer.buffers(100), moe.MoeLayerBuffers) and isinstance(layer.buffers(batch), moe.FewTokenBuffers)
    step = serve._next(x[-batch:], first[-batch:])
    for y in rows:
        logits = (_f64(step) @ _f64(w_router).T).astype(np.float32)
        idx, w, _ = O.route_topk(logits, K, ES, True)
        want, far = M.layer_few(_f64(step), idx, w.astype(np.float64), *values)
        assert (np.abs(_f64(y) - want) <= far).all()
        step = serve._next(step, y)


def test_prompt_is_that_of_the_entry_points(moe, model):
    w_router, weights, x = model
    layer = serve.ServedLayer(w_router, *weights, K, ES)
    buf = moe.MoeLayerBuffers(moe.Shape(100, D, F, E, K, ES), with_backward=False)
    assert torch.equal(layer(x), moe.layer_mxfp4_forward(buf, x, moe.quantize_experts(*weights), w_router=w_router))
    full = serve.ServedLayer(w_router, *weights, K, ES, mxfp4=False)
    assert torch.equal(full(x), moe.layer_forward(buf, x, *weights, w_router=w_router))
    few = moe.FewTokenBuffers(moe.Shape(7, D, F, E, K, ES))
    assert torch.equal(full(x[:7]), moe.layer_few_forward(few, x[:7], weights, w_router=w_router))


def test_refusals(moe, model):
    w_router, weights, x = model
    with pytest.raises(ValueError):
        serve.ServedLayer(w_router, *weights, K, 0)
    layer = serve.ServedLayer(w_router, *weights, K, ES)
    with pytest.raises((ValueError, moe.MoeError)):
        layer(x[:, :128].contiguous())


def test_command(moe, capsys):
    assert serve.main("--dims 256x192 --experts 8 --top-k 2 --shared 1 --prompt 80 --batch 2 --steps 3".split()) == 0
    assert '"step_us"' in capsys.readouterr().out
