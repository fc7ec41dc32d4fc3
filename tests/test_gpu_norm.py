"""Layer norm and RMS norm with the residual sum, and their gradients, against the fp64 definition."""
import numpy as np
import pytest
import torch

from oracle import front_oracle as F

pytestmark = pytest.mark.gpu
U = 2.0 ** -24      # half a step of fp32, relative
HALF = 2.0 ** -8    # of bf16
# A sum over a row: at most 32 values one after another in a lane, 6 steps across lanes, up to 8 wavefronts, and what went before each: 64 U of the sum
# of magnitudes is more than that.
SUM = 64 * U

ROWS_COLS = [(1, 8), (2, 16), (3, 64), (7, 504), (5, 512), (4, 520), (1003, 1088), (13, 2040), (6, 2048), (3, 2056), (1, 4096), (9, 4096), (5, 4104),
             (3, 5120), (4, 7168), (2, 8192), (3, 8200), (2, 16384), (3000, 64), (2100, 520), (1100, 2304)]


def make(rows, cols, seed=0, offset=0.0):
    g = torch.Generator().manual_seed(seed + 1000 * rows + cols)
    n = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, generator=g) * std + mean).bfloat16()  # noqa: E731
    return {"x": n(rows, cols, mean=offset), "addend": n(rows, cols, std=0.5), "gamma": n(cols, std=0.3, mean=1.0), "beta": n(cols, std=0.3), "dy": n(rows, cols)}


def guarded(rows, cols, dtype=torch.bfloat16):
    """A tensor and what lies behind it."""
    t = torch.full((rows * cols + 64,), -7.0, dtype=dtype, device="cuda")
    return t[:rows * cols].view(rows, cols) if cols > 1 else t[:rows], t[rows * cols:]


def f64(t):
    return t.double().cpu().numpy()


def check_fwd(moe, d, rows, cols, centre, addend, gamma, beta, eps=1e-6, in_place=False):
    x = d["x"].cuda()
    a = d["addend"].cuda() if addend else None
    y, behind = guarded(rows, cols)
    total, behind_sum = guarded(rows, cols)
    if in_place:
        total = {"x": x, "addend": a}[in_place]
    mean, behind_mean = guarded(rows, 1, torch.float32)
    rstd, behind_rstd = guarded(rows, 1, torch.float32)
    moe.moe_norm_fwd(centre, eps, x, a, d["gamma"].cuda() if gamma else None, d["beta"].cuda() if beta else None, total if addend else None, y,
                     mean if centre else None, rstd)
    torch.cuda.synchronize()
    assert all((b == -7.0).all() for b in (behind, behind_sum, behind_mean, behind_rstd))
    h = d["x"].float() + d["addend"].float() if addend else d["x"].float()
    h = h.bfloat16()
    if addend:
        assert torch.equal(total.cpu(), h)
    h = f64(h)
    gm, bt = f64(d["gamma"]) if gamma else None, f64(d["beta"]) if beta else None
    want, wm, wr = F.norm_fwd(h, gm, bt, centre, eps)
    level = np.abs(h).mean(1, keepdims=True)
    if centre:
        assert (np.abs(f64(mean) - wm) <= SUM * level[:, 0]).all()
    # the squares' sum, and twice the mean's error times the sum of differences that are not quite zero: second order; rstd takes half of it
    assert (np.abs(f64(rstd) - wr) <= (SUM + (SUM * level[:, 0] * wr) ** 2) * wr).all()
    xh = (h - wm[:, None]) * wr[:, None]
    inner = (np.abs(xh) * 2 * SUM + (SUM * level * wr[:, None] if centre else 0)) * (1 if gm is None else np.abs(gm)) + (0 if bt is None else 2 * U * np.abs(bt))
    off = np.abs(f64(y) - want) - (HALF * (np.abs(want) + inner) + inner)
    assert (off <= 0).all(), off.max()
    return total if addend else x, mean, rstd


def check_bwd(moe, d, rows, cols, centre, addend, gamma, beta, accumulate=False, in_place=None):
    h = d["x"].cuda()
    _, mean, rstd = F.norm_fwd(f64(d["x"]), None, None, centre, 1e-6)
    mean, rstd = torch.from_numpy(mean).float(), torch.from_numpy(rstd).float()
    dy, a = d["dy"].cuda(), d["addend"].cuda() if addend else None
    dx, behind = guarded(rows, cols)
    if in_place:
        dx = {"dy": dy, "addend": a}[in_place]
    grads = [torch.full((cols + 8,), 3.0, device="cuda") for _ in range(2)]
    nbytes = moe.norm_workspace_bytes(rows, cols)
    ws = torch.full((nbytes + 256,), 77, dtype=torch.uint8, device="cuda")
    moe.moe_norm_bwd(centre, dy, h, d["gamma"].cuda() if gamma else None, mean.cuda() if centre else None, rstd.cuda(), a, dx, grads[0],
                     grads[1] if beta else None, accumulate, ws[:nbytes])
    torch.cuda.synchronize()
    assert (behind == -7.0).all() and (ws[nbytes:] == 77).all() and all((g[cols:] == 3.0).all() for g in grads)
    want, wg, wb, size, size_g, size_b = F.norm_bwd(f64(d["dy"]), f64(d["x"]), f64(d["gamma"]) if gamma else None, f64(mean), f64(rstd), centre,
                                                    f64(d["addend"]) if addend else None)
    off = np.abs(f64(dx) - want) - (HALF * np.abs(want) + 3 * SUM * size)
    assert (off <= 0).all(), off.max()
    # a column: a lane's rows one after another (at most rows / blocks of them), then the blocks' parts: 1 / 16 of them in a row, then 16
    turns = rows / 256 + 1100 / 16 + 32
    old = 3.0 if accumulate else 0.0
    assert (np.abs(f64(grads[0][:cols]) - wg - old) <= (turns + 8) * U * (size_g + old)).all()
    if beta:
        assert (np.abs(f64(grads[1][:cols]) - wb - old) <= (turns + 8) * U * (size_b + old)).all()
    else:
        assert (grads[1] == 3.0).all()
    return dx, grads


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("addend,gamma,beta", [(False, True, True), (True, True, False), (True, False, False), (False, False, True)])
@pytest.mark.parametrize("rows,cols", ROWS_COLS)
def test_norm_fwd(moe, rows, cols, addend, gamma, beta, centre):
    check_fwd(moe, make(rows, cols), rows, cols, centre, addend, gamma, beta)


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("addend,gamma,beta", [(False, True, True), (True, True, False), (True, False, True)])
@pytest.mark.parametrize("rows,cols", ROWS_COLS)
def test_norm_bwd(moe, rows, cols, addend, gamma, beta, centre):
    check_bwd(moe, make(rows, cols, 1), rows, cols, centre, addend, gamma, beta)


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("rows,cols", [(19, 128), (19, 136), (35, 256), (35, 264), (9000, 200), (1100, 6200), (1030, 16384), (2100, 4104)])
def test_norm_by_other_lanes_and_launches(moe, rows, cols, centre):
    """Rows of a quarter and half a wavefront, and one row either side of them; many long rows."""
    for addend, beta in ((False, True), (True, False)):
        check_fwd(moe, make(rows, cols, 8), rows, cols, centre, addend, True, beta)
        check_bwd(moe, make(rows, cols, 9), rows, cols, centre, addend, True, beta)


def test_gradient_in_place_of_the_rows(moe):
    """dx over h itself: with the gradients of the weights, which h is read for as well."""
    for rows in (37, 1500):
        d = make(rows, 2304, 10)
        want, grads = check_bwd(moe, d, rows, 2304, False, True, True, True)
        h, (_, _, rstd) = d["x"].cuda(), F.norm_fwd(f64(d["x"]), None, None, False, 1e-6)
        g2 = [torch.empty(2304, device="cuda") for _ in range(2)]
        ws = torch.empty(moe.norm_workspace_bytes(rows, 2304), dtype=torch.uint8, device="cuda")
        moe.moe_norm_bwd(False, d["dy"].cuda(), h, d["gamma"].cuda(), None, torch.from_numpy(rstd).float().cuda(), d["addend"].cuda(), h, *g2, False, ws)
        assert torch.equal(h, want)
        for a, b, x in zip(g2, grads, (f64(d["dy"]) * f64(d["x"]) * rstd[:, None], f64(d["dy"]))):
            # (summed in another order: twice what check_bwd allows one sum)
            assert (np.abs(f64(a) - f64(b[:2304])) <= 2 * (rows / 256 + 1100 / 16 + 40) * U * np.abs(x).sum(0)).all()


def test_offsets_past_32_bits(moe):
    rows, cols = (1 << 22) + 5, 520
    x = torch.randn(1 << 20, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).bfloat16()
    x = torch.cat([x, x * 2, x * 3, x * 4, x[:5] * 5])
    gamma = torch.linspace(0.5, 1.5, cols, device="cuda").bfloat16()
    total, y = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    moe.moe_norm_fwd(True, 1e-6, x, x, gamma, None, total, y, mean, rstd)
    dx = torch.empty_like(x)
    moe.moe_norm_bwd(True, y, total, gamma, mean, rstd, x, dx, None, None, False, None)
    for at in (0, (1 << 20) - 3, (1 << 31) // cols - 4, (1 << 22) - 4, rows - 8):
        some = slice(at, at + 8)
        want = [torch.empty_like(x[some]) for _ in range(3)] + [torch.empty(8, device="cuda") for _ in range(2)]
        moe.moe_norm_fwd(True, 1e-6, x[some], x[some], gamma, None, want[0], want[1], want[3], want[4])
        moe.moe_norm_bwd(True, want[1], want[0], gamma, want[3], want[4], x[some], want[2], None, None, False, None)
        for a, b in zip((total, y, dx, mean, rstd), want):
            assert torch.equal(a[some], b)


@pytest.mark.parametrize("cols", [64, 1088, 4096, 7168])
@pytest.mark.parametrize("offset", [100.0, 1000.0])
def test_rows_far_from_zero(moe, cols, offset):
    """The differences from the mean are what is squared."""
    d = make(9, cols, 2, offset)
    check_fwd(moe, d, 9, cols, True, False, True, True)
    check_bwd(moe, d, 9, cols, True, False, True, True)


@pytest.mark.parametrize("cols", [64, 1088, 4096, 8200])
def test_in_place(moe, cols):
    d = make(37, cols, 3)
    for where in ("x", "addend"):
        check_fwd(moe, d, 37, cols, True, True, True, True, in_place=where)
    for where in ("dy", "addend"):
        check_bwd(moe, d, 37, cols, False, True, True, True, in_place=where)


@pytest.mark.parametrize("cols", [64, 2304, 7168])
def test_accumulates_and_repeats(moe, cols):
    d = make(700, cols, 4)
    first = check_bwd(moe, d, 700, cols, True, True, True, True, accumulate=True)
    again = check_bwd(moe, d, 700, cols, True, True, True, True, accumulate=True)
    assert torch.equal(first[0], again[0]) and all(torch.equal(a, b) for a, b in zip(first[1], again[1]))


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("cols", [64, 520, 4096])
def test_a_row_is_its_own(moe, cols, centre):
    """NaN and infinities stay in their rows; a row of zeros is beta, of equal values too where it is centred."""
    d = make(11, cols, 5)
    clean = make(11, cols, 5)
    d["x"][2, 3], d["x"][5, 0], d["x"][6, cols - 1] = float("nan"), float("inf"), float("-inf")
    d["x"][8], clean["x"][8] = 0.0, 0.0
    if centre:
        d["x"][9], clean["x"][9] = 5.0, 5.0
    y, y2, rstd = (torch.empty(11, cols, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    rstd = torch.empty(11, device="cuda")
    mean = torch.empty(11, device="cuda")
    gamma, beta = d["gamma"].cuda(), d["beta"].cuda()
    moe.moe_norm_fwd(centre, 1e-6, d["x"].cuda(), None, gamma, beta, None, y, mean, rstd)
    moe.moe_norm_fwd(centre, 1e-6, clean["x"].cuda(), None, gamma, beta, None, y2, mean, rstd)
    good = [r for r in range(11) if r not in (2, 5, 6)]
    assert torch.equal(y[good], y2[good]) and torch.isnan(y[2]).all()
    assert not torch.isfinite(y[5]).all() and not torch.isfinite(y[6]).all()
    assert torch.equal(y[8], beta)
    if centre:
        assert torch.equal(y[9], beta)


def test_no_rows(moe):
    e, f = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    grads = [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
    ws = torch.empty(moe.norm_workspace_bytes(0, 64), dtype=torch.uint8, device="cuda")
    moe.moe_norm_fwd(True, 1e-6, e, None, None, None, None, e, f, f)
    moe.moe_norm_bwd(True, e, e, None, f, f, None, e, *grads, True, ws)
    assert all((g == 3.0).all() for g in grads)
    moe.moe_norm_bwd(True, e, e, None, f, f, None, e, *grads, False, ws)
    assert all((g == 0.0).all() for g in grads)


def test_by_differences(moe):
    """dx and dgamma against differences of the definition at the kernel's own inputs."""
    d = make(6, 72, 6)
    dx, grads = check_bwd(moe, d, 6, 72, True, False, True, True)
    x, gm, dy = f64(d["x"]), f64(d["gamma"]), f64(d["dy"])
    rng = np.random.default_rng(0)
    L = lambda a, b: (F.norm_fwd(a, b, None, True, 1e-6)[0] * dy).sum()  # noqa: E731
    for _ in range(4):
        u, v = rng.normal(size=x.shape), rng.normal(size=gm.shape)
        slope = (L(x + 1e-5 * u, gm) - L(x - 1e-5 * u, gm)) / 2e-5
        assert abs(slope - (f64(dx) * u).sum()) <= HALF * np.abs(f64(dx) * u).sum()
        slope = (L(x, gm + 1e-5 * v) - L(x, gm - 1e-5 * v)) / 2e-5
        assert abs(slope - (f64(grads[0][:72]) * v).sum()) <= 1e-4 * np.abs(v).sum()


def test_on_a_stream_of_its_own_and_as_a_graph(moe):
    rows, cols, bf = 200, 2304, torch.bfloat16
    x, a, dy = (torch.empty(rows, cols, dtype=bf, device="cuda") for _ in range(3))
    gamma, beta = torch.ones(cols, dtype=bf, device="cuda"), torch.zeros(cols, dtype=bf, device="cuda")
    ws = torch.empty(moe.norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")

    def outputs():
        return [torch.zeros(rows, cols, dtype=bf, device="cuda") for _ in range(3)] + [torch.zeros(n, device="cuda") for n in (rows, rows, cols, cols)]

    def step(o):
        total, y, dx, mean, rstd, dgamma, dbeta = o
        moe.moe_norm_fwd(True, 1e-5, x, a, gamma, beta, total, y, mean, rstd)
        moe.moe_norm_bwd(True, dy, total, gamma, mean, rstd, y, dx, dgamma, dbeta, False, ws)

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (x, a, dy, gamma, beta):
            t.normal_(generator=g)

    fill(0)
    side, graphs = torch.cuda.Stream(), []
    for _ in range(2):   # (two graphs on one workspace, replayed in order)
        out = outputs()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(out)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(out)
        graphs.append((graph, out))
    for seed in range(1, 5):
        fill(seed)
        want = outputs()
        step(want)
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(u, v) for u, v in zip(out, want))
