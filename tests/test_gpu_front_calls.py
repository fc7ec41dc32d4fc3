"""Calls in front of the experts as a program makes them: whose logits a gradient is of, which rows a command times, which sizes are taken."""
import pytest
import torch

pytestmark = pytest.mark.gpu

T, D, FF, E, K, ES = 100, 128, 192, 16, 4, 1


def make(seed=0):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).bfloat16().cuda()  # noqa: E731
    n = E + ES
    w = (normal(n, D, FF, std=D ** -0.5), normal(n, D, FF, std=D ** -0.5), normal(n, FF, D, std=FF ** -0.5))
    return normal(T, D), normal(T, D), w, torch.randn(T, E, generator=g).cuda(), normal(E, D, std=D ** -0.5), (0.02 * torch.randn(E, generator=g)).cuda()


def test_a_step_routed_by_logits_differentiates_these(moe):
    """Eager without the logits in the backward call, and captured: what the calls one by one give."""
    x, dout, w, logits, w_router, bias = make()
    s, gate = moe.Shape(T, D, FF, E, K, ES), moe.Gate("sigmoid", 4, 2, 2, 2.5)
    one, two = moe.MoeLayerBuffers(s), moe.MoeLayerBuffers(s)
    for buf in (one, two):
        buf.logits.fill_(float("nan"))   # (nobody's)
    moe.layer_forward(one, x, *w, logits=logits, gate=gate, bias=bias)
    moe.layer_backward(one, dout, *w, gate=gate, balance=2.0)
    want = torch.empty(T, E, device="cuda")
    moe.moe_gate_bwd(s, gate, one.dtopk_w, logits, one.topk_idx, one.topk_w, one.counts, 2.0, want, one.balance_loss, one.ws)
    assert torch.isfinite(want).all() and torch.equal(one.dlogits, want)
    step = moe.CapturedLayerStep(two, x, dout, *w, logits=logits, gate=gate, bias=bias, balance=2.0)
    logits.copy_(make(1)[3])
    moe.layer_forward(one, x, *w, logits=logits, gate=gate, bias=bias)
    moe.layer_backward(one, dout, *w, gate=gate, balance=2.0)
    for _ in range(3):
        two.dlogits.zero_()
        step.replay()
        torch.cuda.synchronize()
        for n in ("topk_idx", "topk_w", "out", "dx", "dlogits", "balance_loss", "dw_gate"):
            assert torch.equal(getattr(one, n), getattr(two, n)), n
    with pytest.raises(ValueError, match="not by both"):
        moe.CapturedLayerStep(two, x, dout, *w, logits=logits, w_router=w_router, gate=gate)


@pytest.mark.parametrize("tokens", [3, 300])
@pytest.mark.parametrize("experts,shared,k", [(1024, 1, 8), (1023, 2, 3), (1024, 1, 20), (4, 2 ** 20 - 4, 2)])
def test_all_experts_with_shared_ones_beside_them(moe, tokens, experts, shared, k):
    """The choice, weights and gradients of the experts are those without shared ones; a shared slot has its id and weight 1."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    logits, bias = torch.randn(tokens, experts, device="cuda", generator=g), 0.05 * torch.randn(experts, device="cuda", generator=g)
    gate, ws, got = moe.Gate("sigmoid", scale=2.5), torch.empty(4096, dtype=torch.uint8, device="cuda"), []
    dw = torch.randn(tokens, k, device="cuda", generator=g)
    counts = torch.randint(0, 9, (experts,), dtype=torch.int32, device="cuda", generator=g)
    for es in (0, shared):
        s = moe.Shape(tokens, 64, 64, experts, k, es)
        idx, w = torch.empty(tokens, k + es, dtype=torch.int32, device="cuda"), torch.empty(tokens, k + es, device="cuda")
        dlogits, loss, b = torch.empty(tokens, experts, device="cuda"), torch.empty(1, device="cuda"), bias.clone()
        n = torch.cat([counts, torch.full((es,), tokens, dtype=torch.int32, device="cuda")])
        moe.moe_gate_fwd(s, gate, logits, bias, idx, w)
        moe.moe_gate_bwd(s, gate, torch.cat([dw, torch.ones(tokens, es, device="cuda")], 1), logits, idx, w, n, 0.5, dlogits, loss, ws)
        moe.moe_gate_bias_step(s, n, 0.25, b)
        got.append((idx[:, :k], w[:, :k], dlogits, loss, b))
        assert (idx[:, k:] == torch.arange(experts, experts + es, device="cuda")).all() and (w[:, k:] == 1).all()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_without_counts_the_balance_is_not_read(moe):
    x, dout, w, logits, w_router, bias = make(2)
    s, gate, got = moe.Shape(T, 64, 64, E, K), moe.Gate("sigmoid"), []
    idx, tw, dw = torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty(T, K, device="cuda"), torch.randn(T, K, device="cuda")
    moe.moe_gate_fwd(s, gate, logits, bias, idx, tw)
    for balance in (0.0, float("nan"), float("inf")):
        got.append(torch.empty(T, E, device="cuda"))
        moe.moe_gate_bwd(s, gate, dw, logits, idx, tw, None, balance, got[-1])
    assert torch.isfinite(got[0]).all() and torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("norm,batch", [("rms", 2), ("layer", 70)])
def test_the_command_answers_through_its_norm(moe, monkeypatch, norm, batch):
    """Loads, prompts and steps, timed or compared: every row that is routed is a norm's, whose mean square is 1 (as it is drawn it is off by 0.1)."""
    from paper_2605_05049_amd import serve
    seen, captured, route = [], [], moe.binding.moe_router_gate_fwd

    def watch(shape, gate, x, *rest):
        if torch.cuda.is_current_stream_capturing():
            captured.append(x.shape[0])
        else:
            seen.append(x.float().square().mean(1))
        route(shape, gate, x, *rest)

    monkeypatch.setattr(moe.binding, "moe_router_gate_fwd", watch)
    got = serve.run(256, 192, 8, 2, 1, 80, batch, 3, gate=moe.Gate("sigmoid", 4, 2, 2, 2.5), norm=norm, balance_steps=4)
    # each value is rounded to bf16, by 2^-8 of itself at most, and so its square by 2^-7 (and 2^-16); eps and fp32 are below 1e-5
    assert (torch.cat(seen) - 1).abs().max().item() <= 2.0 ** -7 + 3e-5
    assert captured == [batch] and {v.numel() for v in seen} == {80, batch}
    assert got["step_us"] > 0 and got["prompt_ms"] > 0 and got["off_step"] < 0.5 and got["off_prompt"] < 0.5
    assert got["load_after"] >= 1
