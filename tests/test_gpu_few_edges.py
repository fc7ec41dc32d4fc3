"""The layer for a few tokens at the ends of what its formats hold."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx_oracle as M
from test_gpu_few import Case, _bf16, _f64

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("mx", [False, True], ids=["bf16", "mxfp4"])


def _bits(a):
    return W.f32_to_bf16_bits(np.asarray(a, np.float32))


@BOTH
@pytest.mark.parametrize("T", [2, 20])
@pytest.mark.parametrize("g,u", [((2.0 ** 30, 2.0 ** 30), (2.0 ** 35, 2.0 ** 35)), ((2.0 ** 32 * 1.40625, 2.0 ** 32), (2.0 ** 31 * 1.421875, 2.0 ** 32))],
                         ids=["past fp32", "past bf16"])
def test_hidden_values_past_the_largest(moe, g, u, T, mx):
    """A hidden value that rounds to an infinity is one, and gives infinities of W_down's signs (no NaN).  g, u: a token's value and a weight."""
    d, f = 64, 64
    c = Case(T, d, f, 1, 1, 0, 1, mx)
    x = np.zeros((T, d))
    x[:, 0], x[:, 1] = g[0], u[0]
    c.x = _bits(x)
    wg, wu, wd = np.zeros((1, d, f)), np.zeros((1, d, f)), np.ones((1, f, d))
    wg[0, 0, 5], wu[0, 1, 5] = g[1], u[1]
    wd[0, 5, ::2] = -1.0
    if mx:
        c.weights = [torch.from_numpy(a).cuda() for v in (wg, wu, wd) for a in M.quantize(np.ascontiguousarray(v.transpose(0, 2, 1)))]
    else:
        c.weights = [_bf16(_bits(v)) for v in (wg, wu, wd)]
    out = c.run(moe, (np.zeros((T, 1), np.int32), np.ones((T, 1), np.float32))).out.float().cpu().numpy()
    want = np.where(np.arange(d) % 2 == 0, -np.inf, np.inf)
    assert np.array_equal(out, np.broadcast_to(want, out.shape)), out[0, :4]
