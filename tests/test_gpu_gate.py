"""Routing with softmax or sigmoid scores, a bias and groups, against the fp64 definition: the choice exactly, weights and gradients within what fp32
rounds."""
import numpy as np
import pytest
import torch

from oracle import front_oracle as F

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of fp32, relative

CASES = [
    # T, E, k, groups, kept, best, scores, bias, renorm, Es, scale
    (1, 64, 6, 1, 1, 1, "softmax", False, True, 2, 1.0),
    (1, 1, 1, 1, 1, 1, "sigmoid", True, True, 0, 1.0),
    (5, 4, 4, 1, 1, 1, "softmax", True, False, 0, 1.0),
    (257, 8, 2, 1, 1, 1, "softmax", False, False, 0, 1.0),
    (130, 8, 2, 8, 3, 1, "sigmoid", True, True, 1, 2.5),
    (131, 16, 4, 2, 1, 2, "softmax", True, True, 0, 1.0),
    (63, 60, 4, 6, 3, 1, "softmax", True, False, 1, 1.0),
    (100, 33, 5, 3, 2, 2, "sigmoid", False, True, 0, 1.0),
    (77, 64, 8, 8, 4, 2, "sigmoid", True, True, 0, 2.5),
    (70, 72, 9, 4, 2, 2, "sigmoid", True, True, 0, 1.0),
    (50, 96, 12, 4, 3, 1, "softmax", False, True, 0, 0.5),
    (300, 128, 4, 1, 1, 1, "sigmoid", True, False, 0, 1.0),
    (40, 160, 6, 8, 3, 1, "softmax", True, True, 2, 16.0),
    (517, 256, 8, 8, 4, 2, "sigmoid", True, True, 1, 2.5),
    (33, 256, 8, 8, 4, 2, "sigmoid", False, True, 0, 1.0),
    (33, 256, 8, 16, 4, 2, "softmax", True, True, 0, 1.0),
    (33, 256, 8, 32, 5, 1, "softmax", False, True, 0, 1.0),
    (33, 250, 7, 2, 1, 2, "sigmoid", True, True, 0, 1.0),
    (21, 256, 16, 1, 1, 1, "softmax", False, True, 0, 1.0),
    (21, 256, 17, 1, 1, 1, "sigmoid", True, True, 0, 1.0),
    (9, 257, 8, 1, 1, 1, "sigmoid", True, True, 0, 1.0),
    (9, 512, 8, 8, 4, 2, "sigmoid", True, True, 0, 1.0),
    (7, 516, 3, 12, 4, 2, "softmax", True, True, 0, 1.0),
    (5, 1000, 100, 1, 1, 1, "softmax", True, True, 0, 1.0),
    (4, 1024, 8, 512, 9, 2, "sigmoid", True, True, 0, 1.0),
    (3, 1020, 40, 4, 2, 1, "sigmoid", True, True, 4, 1.0),
]


def make(T, E, seed, mask="none", scale=1.0):
    rng = np.random.default_rng([seed, T, E])
    logits = (scale * rng.normal(size=(T, E)) + 0.5 * rng.normal(size=E)).astype(np.float32)
    bias = (0.05 * rng.normal(size=E)).astype(np.float32)
    if mask == "wild":   # whatever a mask may be made of, in places drawn
        for v in (-np.inf, np.nan, -1e30, -np.finfo(np.float32).max, np.inf, np.finfo(np.float32).max, -0.0, 0.0, -200.0):
            logits[rng.random((T, E)) < 0.08] = v
        logits[::5] = -np.inf
        bias[rng.random(E) < 0.05] = -np.inf
        bias[rng.random(E) < 0.05] = np.nan
    elif mask == "ties":
        logits = rng.choice(np.array([-1.0, 0.0, 0.5, 0.5, 1.0], np.float32), size=(T, E))
        bias = rng.choice(np.array([0.0, 0.0, 0.25], np.float32), size=E)
    elif mask == "near":   # scores plus bias that fp32 cannot tell apart
        s = 1 / (1 + np.exp(-logits[0].astype(np.float64)))
        bias = (0.75 - s).astype(np.float32)
        logits = np.nextafter(logits[0], np.where(rng.random((T, E)) < 0.5, np.inf, -np.inf).astype(np.float32)).astype(np.float32)
    return logits, bias


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def spread(logits, alive_rows=None):
    """How far apart the finite logits of a row lie, at most: the exponentials' arguments."""
    l = np.where(logits > F.MASKED, logits, np.nan).astype(np.float64)
    l = l[~np.isnan(l).all(1)]
    return float(min((np.nanmax(l, 1) - np.nanmin(l, 1)).max(), 200.0)) if len(l) else 0.0


def run_fwd(moe, logits, bias, k, groups, kept, best, scores, renorm, Es, scale, stream=None):
    T, E = logits.shape
    s = moe.Shape(T, 64, 64, E, k, Es, renorm)
    idx = torch.full((T + 1, k + Es), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T + 1, k + Es), -7.0, device="cuda")
    gate = moe.Gate(scores, groups, kept, best, scale)
    moe.moe_gate_fwd(s, gate, gpu(logits), gpu(bias), idx, w, stream)
    torch.cuda.synchronize()
    assert (idx[T] == -7).all() and (w[T] == -7.0).all()   # rows behind the last
    return s, gate, idx[:T], w[:T]


def check_fwd(logits, bias, idx, w, k, groups, kept, best, scores, renorm, Es, scale):
    want_idx, want_w = F.gate_fwd(logits, bias, k, scores, groups, kept, best, renorm, scale, Es)
    assert np.array_equal(idx.cpu().numpy(), want_idx)
    # exp(l - top): the argument is rounded (its size times U) and the function is off by 2 U; up to 10 additions of a lane, 6 across, two divisions
    tol = (2 * spread(logits) + 40) * U
    got = w.cpu().numpy().astype(np.float64)
    assert (np.abs(got - want_w) <= tol * np.abs(want_w) + 1e-37).all(), np.abs(got - want_w).max()
    return want_idx, want_w


@pytest.mark.parametrize("mask", ["none", "wild", "ties", "near"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_gate_fwd(moe, case, mask):
    T, E, k, groups, kept, best, scores, with_bias, renorm, Es, scale = case
    logits, bias = make(T, E, 1, mask)
    bias = bias if with_bias else None
    _, _, idx, w = run_fwd(moe, logits, bias, k, groups, kept, best, scores, renorm, Es, scale)
    check_fwd(logits, bias, idx, w, k, groups, kept, best, scores, renorm, Es, scale)


@pytest.mark.parametrize("case", [
    (2500, 256, 8, 8, 4, 2, "sigmoid"), (2500, 256, 7, 8, 4, 2, "sigmoid"), (2500, 64, 16, 1, 1, 1, "softmax"), (2500, 64, 9, 4, 3, 2, "softmax"),
    (1500, 128, 6, 1, 1, 1, "softmax"), (1500, 128, 8, 1, 1, 1, "softmax"), (1100, 1024, 16, 4, 2, 2, "sigmoid"), (300, 512, 8, 64, 9, 1, "sigmoid"),
    (1100, 44, 8, 11, 5, 1, "softmax"), (3000, 8, 8, 2, 2, 2, "sigmoid"),
    (2500, 256, 4, 8, 4, 2, "sigmoid"), (2500, 64, 4, 1, 1, 1, "softmax"), (1500, 128, 3, 1, 1, 1, "sigmoid"), (1500, 96, 4, 4, 1, 2, "softmax"),
    (1100, 192, 8, 8, 4, 2, "sigmoid"), (1100, 192, 8, 1, 1, 1, "softmax"), (1100, 384, 6, 16, 3, 1, "sigmoid"), (900, 160, 6, 8, 3, 1, "softmax"),
    (2500, 20, 1, 5, 2, 2, "sigmoid")], ids=lambda c: "-".join(str(v) for v in c))
def test_gate_fwd_of_many_tokens_that_fp32_cannot_decide(moe, case):
    T, E, k, groups, kept, best, scores = case
    logits, bias = make(T, E, 11, "near")
    if scores == "softmax":   # (as `near`, of one token's scores)
        s = np.exp(logits[0].astype(np.float64) - logits[0].max())
        bias = (0.75 - s / s.sum()).astype(np.float32)
    _, _, idx, w = run_fwd(moe, logits, bias, k, groups, kept, best, scores, True, 0, 1.0)
    check_fwd(logits, bias, idx, w, k, groups, kept, best, scores, True, 0, 1.0)


def test_offsets_past_32_bits(moe):
    T, E, k = (1 << 24) + 5, 132, 4
    g = torch.Generator(device="cuda").manual_seed(0)
    few = torch.randn(1 << 20, E, device="cuda", generator=g)
    logits = torch.empty(T, E, device="cuda")
    for i in range(17):
        part = logits[i << 20:(i + 1) << 20]
        torch.mul(few[:len(part)], 1.0 + i, out=part)
    bias, gate = 0.1 * torch.randn(E, device="cuda", generator=g), moe.Gate("sigmoid", 4, 2, 2, 1.0)
    idx, w, dlogits = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda"), torch.empty(T, E, device="cuda")
    moe.moe_gate_fwd(moe.Shape(T, 64, 64, E, k), gate, logits, bias, idx, w)
    moe.moe_gate_bwd(moe.Shape(T, 64, 64, E, k), gate, w, logits, idx, w, None, 0.0, dlogits)
    for at in (0, (1 << 31) // E - 4, (1 << 24) - 4, T - 8):
        some = slice(at, at + 8)
        one = [torch.empty(8, k, dtype=torch.int32, device="cuda"), torch.empty(8, k, device="cuda"), torch.empty(8, E, device="cuda")]
        moe.moe_gate_fwd(moe.Shape(8, 64, 64, E, k), gate, logits[some], bias, one[0], one[1])
        moe.moe_gate_bwd(moe.Shape(8, 64, 64, E, k), gate, one[1], logits[some], one[0], one[1], None, 0.0, one[2])
        assert torch.equal(idx[some], one[0])
        # (sums of other lanes' orders)
        assert (w[some] - one[1]).abs().max().item() <= 16 * U and (dlogits[some] - one[2]).abs().max().item() <= 64 * U


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_gate_fwd_of_scores_far_from_even(moe, scores):
    logits, bias = make(64, 128, 2, scale=30.0)
    for b in (None, bias):
        _, _, idx, w = run_fwd(moe, logits, b, 6, 4, 2, 2, scores, True, 0, 1.0)
        check_fwd(logits, b, idx, w, 6, 4, 2, 2, scores, True, 0, 1.0)


@pytest.mark.parametrize("T", [2, 1021, 5000])
def test_gate_fwd_of_many_tokens(moe, T):
    """Every kernel's grid, with a last block that is not full; a sample against the definition, all against a token by itself."""
    logits, bias = make(T, 256, 3)
    args = (8, 8, 4, 2, "sigmoid", True, 0, 2.5)
    _, _, idx, w = run_fwd(moe, logits, bias, *args)
    some = np.unique(np.r_[0, T - 1, np.random.default_rng(0).integers(0, T, 100)])
    check_fwd(logits[some], bias, idx[some.tolist()], w[some.tolist()], *args)
    _, _, one, w1 = run_fwd(moe, logits[T - 1:], bias, *args)
    assert torch.equal(one[0], idx[T - 1]) and torch.equal(w1[0], w[T - 1])


@pytest.mark.parametrize("mask", ["none", "wild"])
@pytest.mark.parametrize("balance", [None, 0.0, 50.0])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_gate_bwd(moe, case, balance, mask):
    T, E, k, groups, kept, best, scores, with_bias, renorm, Es, scale = case
    logits, bias = make(T, E, 5, mask)
    idx, w = F.gate_fwd(logits, bias if with_bias else None, k, scores, groups, kept, best, renorm, scale, Es)
    w = w.astype(np.float32)
    check_bwd(moe, logits, idx, w, k, scores, renorm, scale, Es, balance)


def check_bwd(moe, logits, idx, w, k, scores, renorm, scale, Es, balance, bits=None):
    T, E = logits.shape
    dw = np.random.default_rng(7).normal(size=(T, k + Es)).astype(np.float32)
    counts = None if balance is None else np.bincount(idx.reshape(-1), minlength=E + Es).astype(np.int32)
    s = moe.Shape(T, 64, 64, E, k, Es, renorm)
    dlogits = torch.full((T + 1, E), -7.0, device="cuda")
    loss = torch.full((2,), -7.0, device="cuda") if balance is not None else None
    ws = torch.empty(16384, dtype=torch.uint8, device="cuda") if balance is not None else None
    moe.moe_gate_bwd(s, moe.Gate(scores, scale=scale), gpu(dw), gpu(logits), gpu(idx), gpu(w), gpu(counts), balance or 0.0, dlogits, loss, ws)
    torch.cuda.synchronize()
    assert (dlogits[T] == -7.0).all()
    want, want_loss, size = F.gate_bwd(dw, logits, idx, w, k, scores, renorm, scale, counts, balance or 0.0)
    # terms: exponentials as above; sums over k, then over E, of up to k + 4 and 26 roundings
    tol = (3 * spread(logits) + 2 * k + 60) * U
    got = dlogits[:T].cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= tol * size + 1e-37).all(), (np.abs(got - want) / (size + 1e-30)).max()
    if loss is not None:
        assert loss[1].item() == -7.0
        assert abs(loss[0].item() - want_loss) <= (tol + 100 * U) * abs(want_loss) + 1e-37   # (a block's tokens one after another: up to T / 4096)
    return dlogits[:T]


def test_gate_bwd_of_many_tokens(moe):
    logits, bias = make(20000, 128, 6)
    idx, w = np.argsort(-logits, 1, kind="stable")[:, :4].astype(np.int32), None
    w = F.gate_weights(logits, idx, "sigmoid", True, 2.5).astype(np.float32)
    a = check_bwd(moe, logits, idx, w, 4, "sigmoid", True, 2.5, 0, 0.01)
    assert torch.equal(a, check_bwd(moe, logits, idx, w, 4, "sigmoid", True, 2.5, 0, 0.01))   # the same bits every time


@pytest.mark.parametrize("T,E,k,scores,renorm", [(20000, 130, 4, "softmax", False), (3000, 30, 4, "sigmoid", False), (2000, 1023, 70, "sigmoid", True),
                                                   (5000, 500, 9, "softmax", True), (4100, 36, 2, "softmax", False),
                                                   (3001, 8, 8, "sigmoid", True), (2500, 16, 11, "softmax", True), (700, 12, 3, "softmax", False),
                                                   (511, 4, 1, "sigmoid", False), (2003, 84, 5, "sigmoid", True), (1501, 160, 6, "softmax", False),
                                                   (1001, 320, 4, "softmax", True), (701, 600, 8, "sigmoid", False), (1203, 70, 3, "softmax", False),
                                                   (1203, 97, 3, "sigmoid", True), (1203, 190, 8, "sigmoid", False), (901, 205, 8, "softmax", False),
                                                   (901, 301, 2, "sigmoid", True), (501, 450, 8, "softmax", False), (501, 601, 8, "sigmoid", True)])
def test_gate_bwd_of_many_tokens_of_odd_sizes(moe, T, E, k, scores, renorm):
    logits, _ = make(T, E, 12)
    idx = np.argsort(-logits, 1, kind="stable")[:, :k].astype(np.int32)
    w = F.gate_weights(logits, idx, scores, renorm, 1.5).astype(np.float32)
    check_bwd(moe, logits, idx, w, k, scores, renorm, 1.5, 0, 2.0)


def test_gate_bwd_sums_an_expert_that_is_named_twice(moe):
    logits, _ = make(9, 24, 8)
    idx = np.tile(np.array([3, 3, 7, 3], np.int32), (9, 1))
    w = np.full((9, 4), 0.25, np.float32)
    for scores in ("softmax", "sigmoid"):
        for renorm in (True, False):
            check_bwd(moe, logits, idx, w, 4, scores, renorm, 1.0, 0, None)


def test_gate_by_differences(moe):
    """The gradient of the kernels' own weights, by differences of them in directions drawn (the choice stays)."""
    logits, bias = make(64, 32, 9)
    rng = np.random.default_rng(1)
    for scores in ("softmax", "sigmoid"):
        s, gate, idx, w = run_fwd(moe, logits, bias, 4, 4, 2, 2, scores, True, 0, 1.0)
        dw = torch.from_numpy(rng.normal(size=(64, 4)).astype(np.float32)).cuda()
        d = torch.empty(64, 32, device="cuda")
        moe.moe_gate_bwd(s, gate, dw, gpu(logits), idx.contiguous(), w.contiguous(), None, 0.0, d)
        u = rng.normal(size=logits.shape).astype(np.float32)
        h, L = 2.0 ** -7, []
        same = torch.ones(64, dtype=torch.bool, device="cuda")
        for sign in (1, -1):
            _, _, i2, w2 = run_fwd(moe, logits + np.float32(sign * h) * u, bias, 4, 4, 2, 2, scores, True, 0, 1.0)
            same &= (i2 == idx).all(1)
            L.append((w2.double() * dw.double()).sum(1))
        slope = ((L[0] - L[1]) / (2 * h))[same]
        want = (d.double() * torch.from_numpy(u).cuda().double()).sum(1)[same]
        assert same.sum() > 32
        # third derivatives: h^2 / 6 times |u|^3 |dw| of a few units; the weights' rounding over h
        assert (slope - want).abs().max().item() < 64 * h * h / 6 + 32 * U / h


def test_bias_step(moe):
    E, Es = 100, 3
    s = moe.Shape(64, 64, 64, E, 2, Es)
    rng = np.random.default_rng(2)
    for counts in (rng.integers(0, 40, E + Es), np.full(E + Es, 5), np.full(E + Es, 2 ** 31 - 1), np.r_[np.zeros(E - 1, int), 2 ** 31 - 1, 1, 1, 1]):
        counts = counts.astype(np.int32)
        bias = rng.normal(size=E + 1).astype(np.float32)
        b = gpu(bias)
        moe.moe_gate_bias_step(s, gpu(counts), 0.25, b)
        n = counts[:E].astype(object)
        step = np.array([0.25 if v * E < n.sum() else -0.25 if v * E > n.sum() else 0.0 for v in n], np.float32)
        assert np.array_equal(b.cpu().numpy(), np.r_[bias[:E] + step, bias[E:]])


def test_no_tokens(moe):
    s = moe.Shape(0, 64, 64, 8, 2)
    e, i = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    loss, ws, bias = torch.full((1,), 3.0, device="cuda"), torch.empty(16384, dtype=torch.uint8, device="cuda"), torch.ones(8, device="cuda")
    counts = torch.zeros(8, dtype=torch.int32, device="cuda")
    g = moe.Gate()
    moe.moe_gate_fwd(s, g, e, None, i, e)
    moe.moe_gate_bwd(s, g, e, e, i, e, counts, 1.0, e, loss, ws)
    moe.moe_gate_bias_step(s, counts, 1.0, bias)
    assert loss.item() == 0.0 and (bias == 1).all()


@pytest.mark.parametrize("T,E", [(1, 8), (64, 64), (300, 256), (9000, 40)])
def test_router_gate_is_the_two_calls(moe, T, E):
    d, k = 512, 4
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, d, device="cuda", generator=g).bfloat16()
    w_router = (0.05 * torch.randn(E, d, device="cuda", generator=g)).bfloat16()
    bias = 0.02 * torch.randn(E, device="cuda", generator=g)
    s, gate = moe.Shape(T, d, 64, E, k), moe.Gate("sigmoid", 4, 2, 2, 2.0)
    ws = torch.empty(moe.workspace_bytes(s), dtype=torch.uint8, device="cuda")
    got = [torch.empty(T, E, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")]
    want = [torch.empty_like(v) for v in got]
    moe.moe_router_gate_fwd(s, gate, x, w_router, bias, *got, ws)
    moe.moe_router_fwd(s, x, w_router, want[0], ws)
    moe.moe_gate_fwd(s, gate, want[0], bias, want[1], want[2])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_a_stream_of_its_own_and_as_a_graph(moe):
    """Captured once, replayed with other inputs, eager work and synchronisations in between; two graphs that share a workspace, in order."""
    T, E, k = 300, 64, 6
    s, gate = moe.Shape(T, 64, 64, E, k), moe.Gate("sigmoid", 8, 4, 2, 2.5)
    logits, bias, dw = torch.empty(T, E, device="cuda"), torch.empty(E, device="cuda"), torch.empty(T, k, device="cuda")
    counts = torch.empty(E, dtype=torch.int32, device="cuda")
    ws = torch.empty(16384, dtype=torch.uint8, device="cuda")

    def step(out):
        moe.moe_gate_fwd(s, gate, logits, bias, out["idx"], out["w"])
        moe.moe_gate_bwd(s, gate, dw, logits, out["idx"], out["w"], counts, 0.5, out["dlogits"], out["loss"], ws)

    def outputs():
        return {"idx": torch.zeros(T, k, dtype=torch.int32, device="cuda"), "w": torch.zeros(T, k, device="cuda"),
                "dlogits": torch.zeros(T, E, device="cuda"), "loss": torch.zeros(1, device="cuda")}

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        logits.normal_(generator=g), bias.normal_(std=0.05, generator=g), dw.normal_(generator=g)
        counts.random_(0, 50, generator=g)

    fill(0)
    side, graphs = torch.cuda.Stream(), []
    for _ in range(2):
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
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for name, v in want.items():
                assert torch.equal(out[name], v), name
        other = outputs()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(other)
        side.synchronize()
        assert all(torch.equal(other[n], want[n]) for n in want)
