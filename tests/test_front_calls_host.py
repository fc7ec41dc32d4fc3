"""Host-side checks of which tensors and sizes the calls in front of the experts are given and take."""
import pytest
import torch

import paper_2605_05049_amd as moe
from paper_2605_05049_amd import binding as B

T, D, F, E, K = 3, 64, 64, 8, 2


@pytest.fixture
def calls(monkeypatch):
    """The entry points write down what they are given in place of launching."""
    made = []
    for name in dir(B):
        if name.startswith("moe_"):
            monkeypatch.setattr(B, name, lambda *a, _name=name, **kw: made.append((_name, a)))
    return made


def _layer():
    moe.load_library()
    buf = moe.MoeLayerBuffers(moe.Shape(T, D, F, E, K), device="cpu")
    return buf, torch.zeros(T, D), [torch.zeros(1)] * 3, torch.zeros(T, E), torch.zeros(E, D)


def _logits_of(calls, name, at):
    return [a[at] for n, a in calls if n == name][-1]


def test_the_gates_gradient_is_that_of_the_logits_that_the_forward_call_routed_by(calls):
    buf, x, w, logits, w_router = _layer()
    gate = moe.Gate("sigmoid")
    moe.layer_forward(buf, x, *w, logits=logits, gate=gate)
    moe.layer_backward(buf, x, *w, gate=gate)
    assert _logits_of(calls, "moe_gate_fwd", 2) is logits and _logits_of(calls, "moe_gate_bwd", 3) is logits
    moe.layer_forward(buf, x, *w, w_router=w_router, gate=gate)
    moe.layer_backward(buf, x, *w, gate=gate, x=x, w_router=w_router)
    assert _logits_of(calls, "moe_router_gate_fwd", 5) is buf.logits and _logits_of(calls, "moe_gate_bwd", 3) is buf.logits
    # routed by the caller: what the caller says, or what the router's calls write
    moe.layer_forward(buf, x, *w, logits=logits, gate=gate)
    moe.layer_forward(buf, x, *w)
    moe.layer_backward(buf, x, *w, gate=gate)
    assert _logits_of(calls, "moe_gate_bwd", 3) is buf.logits
    moe.layer_backward(buf, x, *w, gate=gate, logits=logits)
    assert _logits_of(calls, "moe_gate_bwd", 3) is logits
    # without a gate w_router comes first, as ever
    moe.layer_forward(buf, x, *w, logits=logits, w_router=w_router)
    assert calls[-4][0] == "moe_router_route_fwd" and buf.routed_by is buf.logits


def test_a_gate_with_logits_and_a_router_is_refused(calls):
    """Which of the two the backward pass would have to differentiate it could not know."""
    buf, x, w, logits, w_router = _layer()
    for forward in (moe.layer_forward, lambda *a, **kw: moe.layer_mxfp4_forward(*a[:2], a[2:], **kw)):
        with pytest.raises(ValueError, match="not by both"):
            forward(buf, x, *w, logits=logits, w_router=w_router, gate=moe.Gate())
    assert not calls


@pytest.mark.parametrize("E,Es", [(1024, 1), (1023, 2), (4, 1021), (1, 2 ** 20 - 1)])
def test_the_gate_takes_all_its_experts_with_shared_ones_beside_them(E, Es):
    """(No tokens: what is checked is the shape.)  The calls that move rows keep their limit."""
    import ctypes
    lib, shape = moe.load_library(), moe.Shape(0, D, F, E, 1, Es)
    s, g, fake = ctypes.byref(shape._c), ctypes.byref(moe.Gate()._c), ctypes.c_void_p(0x10000)
    assert lib.moe_gate_fwd(s, g, None, None, None, None, None) == 0
    assert lib.moe_gate_bwd(s, g, None, None, None, None, None, 0.0, None, None, None, 0, None) != -2   # (it asks the device for errors)
    assert lib.moe_gate_bias_step(s, fake, 0.1, fake, None) == 0
    assert lib.moe_router_gate_fwd(s, g, None, None, None, None, None, None, None, 0, None) == -2
    assert lib.moe_permute(s, None, fake, None, fake, fake, fake, fake, fake, 1 << 40, None) == -2 and moe.workspace_bytes(shape) == 0
    for bad in (moe.Shape(0, D, F, 1025, 1, 0), moe.Shape(0, D, F, E, 1, 2 ** 20 - E + 1), moe.Shape(0, D, F, E, 1, 2 ** 31 - 1), moe.Shape(0, D, F, E, 1, -1)):
        b = ctypes.byref(bad._c)
        assert lib.moe_gate_fwd(b, g, None, None, None, None, None) == -2 and lib.moe_gate_form(b, g, (ctypes.c_int32 * 4)()) == -2
        assert lib.moe_gate_bias_step(b, fake, 0.1, fake, None) == -2
        assert lib.moe_gate_bwd(b, g, None, None, None, None, None, 0.0, None, None, None, 0, None) == -2


class _On:
    """What the binding asks of a tensor, on a device of its own."""

    def __init__(self, device, dtype, *size):
        self.at, self.dtype, self.size, self.is_cuda, self.device = device, dtype, size, True, torch.device("cuda", device)

    def get_device(self):
        return self.at

    def numel(self):
        n = 1
        for s in self.size:
            n *= s
        return n

    def dim(self):
        return len(self.size)

    shape = property(lambda self: torch.Size(self.size))

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


class _Stream:
    def __init__(self, device):
        self.device_index, self.cuda_stream = device, 0


def _every_call(at, stream):
    """The calls with the tensor `at` on device 1, the others on device 0: (name of the call, how many tensors)."""
    shape, gate = moe.Shape(T, D, F, E, K), moe.Gate()
    f, i, bf, u = torch.float32, torch.int32, torch.bfloat16, torch.uint8

    def tensors(*kinds):
        return [_On(1 if n == at else 0, *kind) for n, kind in enumerate(kinds)]

    idx, w, l, x, row = (i, T, K), (f, T, K), (f, T, E), (bf, T, D), (f, T)
    logits, bias, ti, tw = tensors(l, (f, E), idx, w)
    yield 4, lambda: moe.moe_gate_fwd(shape, gate, logits, bias, ti, tw, stream)
    r = tensors(x, (bf, E, D), (f, E), l, idx, w, (u, 1 << 20))
    yield 7, lambda: moe.moe_router_gate_fwd(shape, gate, *r, stream)
    b = tensors(w, l, idx, w, (i, E), l, (f, 1), (u, 4096))
    yield 8, lambda: moe.moe_gate_bwd(shape, gate, *b[:5], 0.1, *b[5:], stream)
    s = tensors((i, E), (f, E))
    yield 2, lambda: moe.moe_gate_bias_step(shape, s[0], 0.1, s[1], stream)
    n = tensors(x, x, (bf, D), (bf, D), x, x, row, row)
    yield 8, lambda: moe.moe_norm_fwd(True, 1e-6, *n, stream)
    m = tensors(x, x, (bf, D), row, row, x, x, (f, D), (f, D), (u, 1 << 20))
    yield 10, lambda: moe.moe_norm_bwd(True, *m[:9], False, m[9], stream)


@pytest.mark.parametrize("stream", [_Stream(0), None], ids=["stream", "current"])
def test_tensors_on_another_device_than_the_current_one_are_refused(monkeypatch, stream):
    """Each of them, in the first call of a process too, whether a stream is given or not; nothing is launched."""
    launched = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: launched.append(name) or 0

    monkeypatch.setattr(B, "_lib", Library())
    monkeypatch.setattr(B, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    for call, (tensors, _) in enumerate(_every_call(-1, stream)):
        for at in range(tensors):
            monkeypatch.setattr(B, "_device", None)   # (as in a call that no other one came before)
            with pytest.raises(ValueError, match="device 1"):
                list(_every_call(at, stream))[call][1]()
    assert not launched
    for _, fn in _every_call(-1, stream):
        fn()
    assert len(launched) == 6
    if stream is not None:
        for _, fn in _every_call(-1, _Stream(1)):
            with pytest.raises(ValueError, match="stream on device 1"):
                fn()


@pytest.mark.parametrize("balance", [float("nan"), float("inf"), -float("inf")])
def test_without_counts_the_balance_is_not_read(balance):
    """(No tokens: what is checked is the number.)"""
    import ctypes
    lib, s, g = moe.load_library(), ctypes.byref(moe.Shape(0, D, F, E, K)._c), ctypes.byref(moe.Gate()._c)
    fake = ctypes.c_void_p(0x10000)
    assert lib.moe_gate_bwd(s, g, None, None, None, None, None, balance, None, None, None, 0, None) != -2   # (without a device it says so)
    assert lib.moe_gate_bwd(s, g, None, None, None, None, fake, balance, None, None, None, 0, None) == -2
