"""Host-side checks of the entry points for answering: what they refuse, before anything is launched."""
import ctypes
import os
import re

import pytest

import paper_2605_05049_amd as moe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(0x10000)        # aligned, never dereferenced: every call below fails its host checks first
ODD = ctypes.c_void_p(0x10004)
NULL, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    return moe.load_library()


def _with(args, i, v):
    args = list(args)
    args[i] = v
    return args


def test_quantise_refusals(lib):
    for fn, sizes in ((lib.moe_mxfp4_quantize, (4, 64)), (lib.moe_mxfp4_quantize_t, (2, 64, 64))):
        good = [FAKE, *sizes, FAKE, FAKE, None]
        for i in (0, len(good) - 3, len(good) - 2):
            assert fn(*_with(good, i, None)) == NULL
            assert fn(*_with(good, i, ODD)) == ALIGN
        for i in range(1, 1 + len(sizes)):
            assert fn(*_with(good, i, -32)) == SHAPE
    assert lib.moe_mxfp4_quantize(FAKE, 4, 48, FAKE, FAKE, None) == SHAPE            # not whole blocks
    assert lib.moe_mxfp4_quantize(FAKE, 2 ** 32, 32, FAKE, FAKE, None) == SHAPE      # over 2^36 values
    assert lib.moe_mxfp4_quantize_t(FAKE, 1, 48, 64, FAKE, FAKE, None) == SHAPE
    assert lib.moe_mxfp4_quantize_t(FAKE, 1, 64, 12, FAKE, FAKE, None) == SHAPE
    assert lib.moe_mxfp4_quantize_t(FAKE, 65536, 64, 64, FAKE, FAKE, None) == SHAPE
    good = [FAKE, FAKE, 4, 64, FAKE, None]
    for i in (0, 1, 4):
        assert lib.moe_mxfp4_dequantize(*_with(good, i, None)) == NULL
        assert lib.moe_mxfp4_dequantize(*_with(good, i, ODD)) == ALIGN
    assert lib.moe_mxfp4_dequantize(*_with(good, 3, 33)) == SHAPE
    # nothing to do is no error, whatever the pointers
    assert lib.moe_mxfp4_quantize(None, 0, 64, None, None, None) == 0


def test_product_refusals(lib):
    good = [2, 10, 64, 64, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None]
    for i in range(4, 10):
        assert lib.moe_mxfp4_grouped_gemm(*_with(good, i, None)) == NULL
    for i in (4, 5, 7, 8, 9):
        assert lib.moe_mxfp4_grouped_gemm(*_with(good, i, ODD)) == ALIGN
    for i, v in ((0, 0), (0, 1025), (1, -1), (1, 2 ** 31), (2, 60), (2, 0), (2, 2 ** 22 + 8), (3, 48), (3, 0), (3, 2 ** 22 + 32)):
        assert lib.moe_mxfp4_grouped_gemm(*_with(good, i, v)) == SHAPE, (i, v)
    s = moe.Shape(16, 128, 64, 4, 2)
    good = [ctypes.byref(s._c), FAKE, FAKE, *[FAKE] * 6, FAKE, FAKE, 1 << 40, None]
    for i in range(1, 11):
        assert lib.moe_mxfp4_grouped_ffn_fwd(*_with(good, i, None)) == NULL
    assert lib.moe_mxfp4_grouped_ffn_fwd(*_with(good, 3, ODD)) == ALIGN
    assert lib.moe_mxfp4_grouped_ffn_fwd(*_with(good, 10, ctypes.c_void_p(0x10010))) == ALIGN
    assert lib.moe_mxfp4_grouped_ffn_fwd(*_with(good, 11, 256)) == WORKSPACE
    bad = moe.Shape(16, 100, 64, 4, 2)
    assert lib.moe_mxfp4_grouped_ffn_fwd(*_with(good, 0, ctypes.byref(bad._c))) == SHAPE


@pytest.mark.parametrize("name,weights", [("moe_layer_few_fwd", 3), ("moe_layer_few_mxfp4_fwd", 6)])
def test_few_tokens_refusals(lib, name, weights):
    fn = getattr(lib, name)
    s = moe.Shape(16, 128, 64, 4, 2)
    good = [ctypes.byref(s._c), FAKE, FAKE, *[FAKE] * weights, FAKE, FAKE, FAKE, FAKE, 1 << 40, None]
    for i in range(len(good) - 2):
        if i != 2:   # (no router: rows that arrive routed)
            assert fn(*_with(good, i, None)) == NULL, i
        if i > 0:
            assert fn(*_with(good, i, ODD)) == ALIGN, i
    assert fn(*_with(good, len(good) - 3, ctypes.c_void_p(0x10010))) == ALIGN
    assert fn(*_with(good, len(good) - 2, moe.layer_few_workspace_bytes(s) - 1)) == WORKSPACE
    for bad in (moe.Shape(65, 128, 64, 4, 2), moe.Shape(64, 128, 64, 128, 65), moe.Shape(16, 100, 64, 4, 2), moe.Shape(16, 128, 64, 4, 5),
                moe.Shape(-1, 128, 64, 4, 2)):
        assert fn(*_with(good, 0, ctypes.byref(bad._c))) == SHAPE
        assert moe.layer_few_workspace_bytes(bad) == 0


def test_limits_and_workspaces(lib):
    header = open(os.path.join(ROOT, "include", "moe.h")).read()
    assert int(re.search(r"#define MOE_FEW_TOKENS_MAX (\d+)", header).group(1)) == moe.FEW_TOKENS_MAX == 64
    for T in (1, 16, 17, 64):
        n = moe.layer_few_workspace_bytes(moe.Shape(T, 2048, 1408, 64, 6, 2))
        assert n > 0 and n % 256 == 0
    # the 4-bit product's own rows are part of the layer's workspace, which does not grow for them
    s = moe.Shape(256, 512, 1024, 8, 2)
    assert moe.workspace_bytes(s) >= s.N * (512 + 1024) * 17 // 32


def test_binding_refusals(lib):
    import torch
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        moe.moe_mxfp4_quantize(x, u8(4, 32), u8(4, 2))          # host tensors
    with pytest.raises(ValueError):
        moe.FewTokenBuffers(moe.Shape(65, 64, 64, 4, 2), device="cpu")
