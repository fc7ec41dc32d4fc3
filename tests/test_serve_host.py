"""Host-side checks of a layer that only answers: what it refuses, and what it keeps."""
import ctypes

import pytest
import torch

import paper_2605_05049_amd as moe
from paper_2605_05049_amd import serve

E, K, ES, D, F = 8, 2, 1, 128, 192


def _weights():
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    return z(E, D), [z(E + ES, D, F), z(E + ES, D, F), z(E + ES, F, D)]


def _layer():
    moe.load_library()
    w_router, weights = _weights()
    return serve.ServedLayer(w_router, *weights, K, ES, mxfp4=False)


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("mxfp4", [False, True])
def test_weights_of_other_shapes_are_refused(which, mxfp4):
    """Element counts alone would let a transposed matrix pass, to be quantised along the wrong axis."""
    w_router, weights = _weights()
    for wrong in (weights[which].transpose(1, 2).contiguous(), weights[which][:E].contiguous(), weights[which][0]):
        bad = list(weights)
        bad[which] = wrong
        with pytest.raises(ValueError, match="w_gate" if which == 0 else "w_up" if which == 1 else "w_down"):
            serve.ServedLayer(w_router, *bad, K, ES, mxfp4=mxfp4)


@pytest.mark.parametrize("T", [4, 100])
def test_rows_of_another_width_are_refused(T):
    """... also wider ones, of which the calls would take the first T * d_model elements."""
    layer = _layer()
    for x in (torch.zeros(T, 2 * D, dtype=torch.bfloat16), torch.zeros(T, D // 2, dtype=torch.bfloat16), torch.zeros(T * D, dtype=torch.bfloat16),
              torch.zeros(T, 1, D, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match=rf"expected \[T, {D}\]"):
            layer(x)


@pytest.mark.parametrize("args", ["--steps 0", "--steps -3", "--batch 0", "--batch 9 --prompt 8", "--dims 2048", "--dims 2048xwide", "--dims 100x64", "--experts 4 --top-k 5",
                                  "--shared -1"])
def test_command_refuses(args, capsys):
    """As errors of the command line, before anything is made."""
    with pytest.raises(SystemExit) as e:
        serve.main(args.split())
    assert e.value.code == 2 and "error: --" in capsys.readouterr().err


def _held(layer):
    """Bytes of the tensors that a layer keeps beside its weights."""
    seen, todo, found = set(), [layer], {}
    while todo:
        o = todo.pop()
        if id(o) in seen:
            continue
        seen.add(id(o))
        if isinstance(o, torch.Tensor):
            found[o.untyped_storage().data_ptr()] = o.untyped_storage().nbytes()
        elif isinstance(o, dict):
            todo += o.values()
        elif isinstance(o, (list, tuple, set)):
            todo += o
        elif hasattr(o, "__dict__"):
            todo += vars(o).values()
    for w in (layer.w_router, *layer.weights):
        found.pop(w.untyped_storage().data_ptr())
    return sum(found.values())


def test_prompts_of_many_lengths_keep_the_memory_of_the_longest():
    layer = _layer()
    layer.buffers(2000)
    longest = _held(layer)
    for T in (65, 100, 1999, 700, 66, 2000):
        s = layer.buffers(T)
        assert s.shape.T == T and s.out.shape == (T, D) and s.topk_idx.shape == (T, K + ES) and s.x_perm.shape == (T * (K + ES), D)
        assert all(t.is_contiguous() and t.storage_offset() * t.itemsize % 256 == 0 for t in vars(s).values() if isinstance(t, torch.Tensor))
        assert _held(layer) <= longest
    fresh = _layer()
    for T in range(65, 500, 29):   # ever longer ones
        fresh.buffers(T)
    only = _layer()
    only.buffers(T)
    assert _held(fresh) == _held(only)


def test_buffers_of_few_tokens_stay():
    """... for each count, at most 64 of them: a step's graph is replayed on them."""
    layer = _layer()
    first = [layer.buffers(T) for T in (1, 7, 64)]
    layer.buffers(300)
    assert [layer.buffers(T) for T in (1, 7, 64)] == first and all(isinstance(b, moe.FewTokenBuffers) for b in first)


def test_memory_of_a_prompt_on_4_bit_weights():
    """The rows before and after the experts, the rows and H in 4 bits, and the maps: nothing that only a backward or bf16 weights need."""
    for T, d, f, e, k, es in ((4096, 2048, 1408, 64, 6, 2), (8192, 4096, 14336, 8, 2, 0), (65, 64, 64, 1024, 8, 0)):
        s = moe.Shape(T, d, f, e, k, es)
        buf = moe.PromptMemory("cpu", mxfp4=True).buffers(s)
        rows, codes = 2 * s.N * d * 2, s.N * (d + f) * 17 // 32
        maps = 4 * (4 * s.N + 2 * T * e + 2 * s.E_total) + 4 * (s.N + (s.N // 1024 + 1) * s.E_total)   # (the last two: the permutation's scratch)
        assert buf.x_perm.untyped_storage().nbytes() <= rows + codes + maps + 64 * 256
        assert buf.save_g is None and buf.save_u is None
    plain = moe.PromptMemory("cpu").buffers(s)
    assert plain.save_g is None and plain.ws.numel() == moe.workspace_bytes(s)


def test_workspace_of_the_forward_on_4_bit_weights():
    lib = moe.load_library()
    s = moe.Shape(256, 512, 1024, 8, 2)
    n = moe.mxfp4_workspace_bytes(s)
    assert s.N * (512 + 1024) * 17 // 32 <= n < moe.workspace_bytes(s) and n % 256 == 0
    assert moe.mxfp4_workspace_bytes(moe.Shape(256, 500, 1024, 8, 2)) == 0
    fake = ctypes.c_void_p(0x10000)   # (never dereferenced: the call fails its host checks)
    call = lambda size: lib.moe_mxfp4_grouped_ffn_fwd(ctypes.byref(s._c), *[fake] * 10, size, None)  # noqa: E731
    assert call(n - 1) == -4
    many = moe.Shape(4000, 64, 64, 1024, 2)   # the permutation's scratch: 8 x 1024 and 8000 ints
    perm = lambda size: lib.moe_permute(ctypes.byref(many._c), *[fake] * 8, size, None)  # noqa: E731
    assert perm(4 * (8 * 1024 + 8000) - 1) == -4


def test_prompt_memory_of_several_shapes():
    """Shapes with as many tokens have buffers of their own sizes."""
    memory = moe.PromptMemory("cpu")
    a, b, c = moe.Shape(100, 128, 192, 8, 2), moe.Shape(100, 256, 64, 4, 3, 1), moe.Shape(100, 128, 192, 8, 2, 0, 0)
    for s in (a, b, c, a, b):
        buf = memory.buffers(s)
        assert buf.out.shape == (100, s.d_model) and buf.x_perm.shape == (s.N, s.d_model) and buf.shape.renorm == s.renorm
        assert buf.ws.numel() == moe.workspace_bytes(s)
