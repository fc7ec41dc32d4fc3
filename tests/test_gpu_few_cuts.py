"""The layer for a few tokens where a block's part of the contraction takes several fills of its LDS, and where wide columns are taken: many experts, of
which three have the tokens (the others' weights are NaN: nothing may come of them)."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as M

import workloads as W

pytestmark = pytest.mark.gpu

IDS = (2, 31, 39)


def _run(moe, T, d, f, E, k, mx, counts):
    """Slots in turn to the three experts, `counts` of T * k each at least."""
    rng = np.random.default_rng([T, d, f, E, k])
    bf16 = lambda a: W.f32_to_bf16_bits(a.astype(np.float32))  # noqa: E731
    f64 = lambda bits: W.bf16_bits_to_f32(bits).astype(np.float64)  # noqa: E731
    to_gpu = lambda bits: torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
    x = bf16(rng.standard_normal((T, d)))
    local = np.concatenate([np.full(c, i) for i, c in enumerate(counts)] + [np.full(T * k - sum(counts), 2)])
    local = rng.permutation(local).reshape(T, k)
    w = rng.random((T, k)).astype(np.float32)
    values, weights = [], []
    for shape, std in (((3, d, f), 1.5 / np.sqrt(d)), ((3, d, f), 1.5 / np.sqrt(d)), ((3, f, d), 1 / np.sqrt(f))):
        bits = bf16(rng.standard_normal(shape) * std)
        if mx:
            packed = M.quantize(np.ascontiguousarray(f64(bits).transpose(0, 2, 1)))
            values.append(M.dequantize(*packed).transpose(0, 2, 1))
            for a, fill in zip(packed, (0, 255)):
                t = torch.full((E, *a.shape[1:]), fill, dtype=torch.uint8, device="cuda")
                t[list(IDS)] = torch.from_numpy(a).cuda()
                weights.append(t)
        else:
            values.append(f64(bits))
            t = torch.full((E, *bits.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")
            t[list(IDS)] = to_gpu(bits)
            weights.append(t)
    buf = moe.FewTokenBuffers(moe.Shape(T, d, f, E, k))
    buf.topk_idx.copy_(torch.from_numpy(np.asarray(IDS, np.int32)[local]))
    buf.topk_w.copy_(torch.from_numpy(w))
    buf.ws.fill_(0xFF)
    got = moe.layer_few_forward(buf, to_gpu(x), weights).float().cpu().numpy()
    want, far = M.layer_few(f64(x), local, w.astype(np.float64), *values)
    assert (np.abs(got - want) <= far).all(), float((np.abs(got - want) / far).max())


@pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])
@pytest.mark.parametrize("T,d,f,E,k,counts", [
    (64, 4032, 576, 128, 8, (1, 33)),     # d in several fills, its end inside a step of 256; 512 slots
    (64, 576, 4032, 128, 8, (17, 64)),    # d_ffn in several fills
    (64, 2048, 64, 400, 8, (16, 32)),     # two fills of narrow columns
    (40, 1088, 1088, 64, 4, (5, 31)),     # wide columns of bf16 weights, 17 to 64 tokens
    (16, 1088, 1088, 64, 4, (3, 15)),     # ... and at most 16, more than 16 slots of one expert
    (1, 4032, 2048, 40, 3, (1, 1)),       # one token
])
def test_cuts(moe, T, d, f, E, k, counts, mx):
    _run(moe, T, d, f, E, k, mx, counts)
