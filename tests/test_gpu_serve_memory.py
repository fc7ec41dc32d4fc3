"""Whose memory a layer that only answers takes, and when it may be taken again."""
import pytest
import torch

from paper_2605_05049_amd import serve

pytestmark = pytest.mark.gpu

E, K, ES, D, F = 8, 2, 1, 256, 448


def _weights(seed=0):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: (torch.randn(*s, generator=g) * s[-2] ** -0.5).bfloat16().cuda()  # noqa: E731
    return normal(E, D), [normal(E + ES, D, F), normal(E + ES, D, F), normal(E + ES, F, D)]


def _pool(t):
    """The stream whose pool a tensor's memory is from."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not the allocator's")


def test_codes_are_made_in_memory_of_their_stream(moe):
    """Memory of the current stream's pool may still be read by what it had enqueued before; the weights may go as soon as the call returns."""
    _, weights = _weights()
    want = [t.clone() for t in moe.quantize_experts(*weights)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)   # (some 50 ms)
    got = moe.quantize_experts(*weights, stream=side)
    assert all(_pool(t) == side.cuda_stream for t in got)
    old = {w.untyped_storage().data_ptr() for w in weights}
    sizes = [tuple(w.shape) for w in weights]
    del weights
    again = [torch.zeros(*s, dtype=torch.bfloat16, device="cuda") for s in sizes]
    assert not side.query(), "the stream was to be busy until here"
    assert not old & {t.data_ptr() for t in again}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T", [5, 100])
def test_buffers_are_made_in_memory_of_the_calls_stream(moe, T):
    w_router, weights = _weights()
    x = torch.randn(T, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    want = serve.ServedLayer(w_router, *weights, K, ES)(x).clone()
    layer = serve.ServedLayer(w_router, *weights, K, ES)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = layer(x, stream=side)
    assert _pool(out) == _pool(layer.buffers(T).ws) == side.cuda_stream
    side.synchronize()
    assert torch.equal(out, want)
    # ... and on another stream later: what the layer frees waits for that one too
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(100_000_000)
        busy = torch.cuda.current_stream()
        layer(x)
    buffers = {layer.buffers(T).ws.data_ptr(), layer.weights[0].data_ptr()}
    shapes = [(layer.buffers(T).ws.shape, side), (layer.weights[0].shape, torch.cuda.current_stream())]
    del layer, out
    again = []
    for shape, stream in shapes:
        with torch.cuda.stream(stream):
            again.append(torch.empty(shape, dtype=torch.uint8, device="cuda"))
    assert not busy.query(), "the stream was to be busy until here"
    assert not buffers & {t.data_ptr() for t in again}
    torch.cuda.synchronize()
