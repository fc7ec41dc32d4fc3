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


@pytest.mark.parametrize("mxfp4", [False, True], ids=["bf16", "mxfp4"])
def test_prompts_of_many_lengths(moe, mxfp4):
    """One after another, shorter and longer: each answer is right and stays, and the memory is that of the longest."""
    w_router, weights = _weights()
    layer = serve.ServedLayer(w_router, *weights, K, ES, mxfp4=mxfp4)
    x = torch.randn(700, D, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    lengths = (100, 65, 300, 64, 299, 700, 66, 300, 100)
    answers = [layer(x[:T]) for T in lengths]
    for T, got in zip(lengths, answers):
        want = serve.ServedLayer(w_router, *weights, K, ES, mxfp4=mxfp4)(x[:T])
        assert torch.equal(got, want), T
    del answers, got, want
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for T in range(65, 700, 31):
        layer(x[:T])
    assert torch.cuda.memory_allocated() <= held + (1 << 20)


def test_captured_prompts_keep_their_memory(moe):
    """A longer prompt takes another block; the graph's stays its own."""
    w_router, weights = _weights()
    layer = serve.ServedLayer(w_router, *weights, K, ES)
    xs = [torch.randn(90, D, generator=torch.Generator().manual_seed(i)).bfloat16().cuda() for i in range(3)]
    eager = [layer(x) for x in xs]
    static = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(static)
    used = layer._prompts.block.data_ptr()
    layer(torch.cat(xs * 4))
    assert layer._prompts.block.data_ptr() != used
    filler = [torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda") for _ in range(64)]
    for x, want in list(zip(xs, eager)) * 2:
        static.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all((t == 255).all() for t in filler)


@pytest.mark.parametrize("T,d,f,E,k", [(65, 64, 64, 1024, 8), (100, 256, 448, 8, 2), (1500, 320, 64, 300, 3), (3000, 64, 192, 16, 4), (1, 128, 64, 4, 2)])
def test_the_smaller_workspace_is_enough(moe, T, d, f, E, k):
    """Router, permutation and 4-bit FFN with mxfp4_workspace_bytes exactly: the same answers, and nothing written past it."""
    g = torch.Generator().manual_seed(T)
    normal = lambda *s: (torch.randn(*s, generator=g) * s[-2] ** -0.5).bfloat16().cuda()  # noqa: E731
    w_router, weights = normal(E, d), moe.quantize_experts(normal(E, d, f), normal(E, d, f), normal(E, f, d))
    x = normal(T, d)
    s = moe.Shape(T, d, f, E, k)
    n = moe.mxfp4_workspace_bytes(s)
    full, small = moe.MoeLayerBuffers(s, with_backward=False), moe.MoeLayerBuffers(s, with_backward=False, with_saved=False, mxfp4=True)
    assert small.ws.numel() == max(n, 256)
    room = torch.full((n + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
    small.ws = room[:n]
    full.ws.fill_(0xFF)
    want = moe.layer_mxfp4_forward(full, x, weights, w_router=w_router)
    got = moe.layer_mxfp4_forward(small, x, weights, w_router=w_router)
    assert torch.equal(got, want) and torch.equal(small.row_of_slot, full.row_of_slot)
    assert (room[n:] == 0xA5).all()


def test_no_tokens(moe):
    w_router, weights = _weights()
    for mxfp4 in (False, True):
        layer = serve.ServedLayer(w_router, *weights, K, ES, mxfp4=mxfp4)
        assert layer(torch.empty(0, D, dtype=torch.bfloat16, device="cuda")).shape == (0, D)
