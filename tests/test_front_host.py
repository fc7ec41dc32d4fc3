"""Host-side checks of routing and norm in front of the experts: what they refuse, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2605_05049_amd as moe
from paper_2605_05049_amd import binding as B
from paper_2605_05049_amd import serve

FAKE = ctypes.c_void_p(0x10000)        # aligned, never dereferenced: every call below fails its host checks first
ODD = ctypes.c_void_p(0x10004)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return moe.load_library()


def sp(**kw):
    return ctypes.byref(moe.Shape(**{**dict(T=256, d_model=512, d_ffn=1024, E=8, k=2, E_shared=0, renorm=1), **kw})._c)


def gp(*a, **kw):
    return ctypes.byref(moe.Gate(*a, **kw)._c)


def every_gate_call(lib, shape, gate):
    return (lib.moe_gate_fwd(shape, gate, FAKE, None, FAKE, FAKE, None),
            lib.moe_router_gate_fwd(shape, gate, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, 16, None),
            lib.moe_gate_bwd(shape, gate, FAKE, FAKE, FAKE, FAKE, None, 0.0, FAKE, None, None, 0, None))


@pytest.mark.parametrize("gate", [
    dict(groups=3), dict(groups=0), dict(groups=-8), dict(groups=16), dict(groups=4, groups_kept=0), dict(groups=4, groups_kept=5),
    dict(groups=8, groups_kept=1), dict(groups=8, group_best=2), dict(group_best=0), dict(group_best=3), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("inf")), dict(scale=float("nan"))], ids=str)
def test_gates_that_are_refused(lib, gate):
    fields = {**dict(scores="softmax", groups=1, groups_kept=1, group_best=1, scale=1.0), **gate}
    if "groups_kept" not in gate:
        fields["groups_kept"] = max(1, fields["groups"])
    assert set(every_gate_call(lib, sp(), gp(**fields))) == {-2}


def test_gate_refusals(lib):
    g = gp("sigmoid", 4, 2, 2)
    assert set(every_gate_call(lib, sp(k=9), g)) == {-2} and set(every_gate_call(lib, sp(k=5), g)) == {-2}   # more than the groups that stay have
    assert set(every_gate_call(lib, None, g)) == {-1} and set(every_gate_call(lib, sp(), None)) == {-1}
    bad = B._CGate(2, 1, 1, 1, 1.0)
    assert set(every_gate_call(lib, sp(), ctypes.byref(bad))) == {-2}
    s = sp()
    assert lib.moe_gate_fwd(s, g, None, None, FAKE, FAKE, None) == -1
    assert lib.moe_gate_fwd(s, g, FAKE, None, None, FAKE, None) == -1
    assert lib.moe_gate_fwd(s, g, FAKE, None, FAKE, None, None) == -1
    for i in range(4):
        a = [FAKE] * 4
        a[i] = ODD
        assert lib.moe_gate_fwd(s, g, *a, None) == -3
    ok = [FAKE, FAKE, None, FAKE, FAKE, FAKE]
    for i, (put, want) in {0: (None, -1), 1: (None, -1), 2: (ODD, -3), 3: (ODD, -3), 4: (None, -1), 5: (ODD, -3)}.items():
        assert lib.moe_router_gate_fwd(s, g, *(put if j == i else v for j, v in enumerate(ok)), FAKE, BIG, None) == want, i
    assert lib.moe_router_gate_fwd(s, g, *ok, None, BIG, None) == -1
    assert lib.moe_router_gate_fwd(s, g, *ok, FAKE, 16, None) == -4
    assert lib.moe_router_gate_fwd(s, g, *ok, ctypes.c_void_p(0x10010), BIG, None) == -3

    def bwd(dw=FAKE, logits=FAKE, idx=FAKE, w=FAKE, counts=FAKE, balance=0.1, dlogits=FAKE, loss=FAKE, ws=FAKE, n=1 << 12):
        return lib.moe_gate_bwd(s, g, dw, logits, idx, w, counts, balance, dlogits, loss, ws, n, None)

    for name in ("dw", "logits", "idx", "w", "dlogits", "counts", "ws"):
        assert bwd(**{name: None}) == -1, name       # (the loss needs counts and a workspace)
    for name in ("dw", "logits", "idx", "w", "dlogits", "counts", "loss"):
        assert bwd(**{name: ODD}) == -3, name
    assert bwd(ws=ctypes.c_void_p(0x10010)) == -3 and bwd(n=4095) == -4
    assert bwd(balance=float("nan")) == -2 and bwd(balance=float("inf")) == -2
    assert lib.moe_gate_bias_step(s, None, 0.1, FAKE, None) == -1 and lib.moe_gate_bias_step(s, FAKE, 0.1, None, None) == -1
    assert lib.moe_gate_bias_step(s, ODD, 0.1, FAKE, None) == -3 and lib.moe_gate_bias_step(s, FAKE, 0.1, ODD, None) == -3
    for rate in (-0.1, float("nan"), float("inf")):
        assert lib.moe_gate_bias_step(s, FAKE, rate, FAKE, None) == -2


def test_norm_refusals(lib):
    def fwd(rows=4, cols=64, centre=1, eps=1e-6, **put):
        a = {**dict.fromkeys(("x", "addend", "gamma", "beta", "sum", "y", "mean", "rstd"), FAKE), **put}
        return lib.moe_norm_fwd(rows, cols, centre, eps, *a.values(), None)

    def bwd(rows=4, cols=64, centre=1, ws=FAKE, n=BIG, **put):
        a = {**dict.fromkeys(("dy", "h", "gamma", "mean", "rstd", "dx_addend", "dx", "dgamma", "dbeta"), FAKE), **put}
        return lib.moe_norm_bwd(rows, cols, centre, *a.values(), 0, ws, n, None)

    for sizes in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=-8), dict(cols=4), dict(cols=60), dict(cols=moe.NORM_COLS_MAX + 8)):
        assert fwd(**sizes) == -2 and bwd(**sizes) == -2
        assert moe.norm_workspace_bytes(sizes.get("rows", 4), sizes.get("cols", 64)) == 0
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert fwd(eps=eps) == -2
    assert fwd(x=None) == -1 and fwd(y=None) == -1
    assert all(fwd(**{n: ODD}) == -3 for n in ("x", "addend", "gamma", "beta", "sum", "y", "mean", "rstd"))
    assert all(bwd(**{n: None}) == -1 for n in ("dy", "h", "mean", "rstd", "dx", "ws"))
    assert all(bwd(**{n: ODD}) == -3 for n in ("dy", "h", "gamma", "mean", "rstd", "dx_addend", "dx", "dgamma", "dbeta"))
    assert bwd(ws=ctypes.c_void_p(0x10010)) == -3 and bwd(n=moe.norm_workspace_bytes(4, 64) - 1) == -4
    assert moe.norm_workspace_bytes(4, 64) > 0 and moe.norm_workspace_bytes(0, 64) > 0


def test_gate_objects():
    with pytest.raises(ValueError):
        moe.Gate("relu")
    g = moe.Gate("sigmoid", 8)
    assert (g.groups, g.groups_kept, g.group_best, g.scale) == (8, 8, 1, 1.0)
    with pytest.raises(AttributeError):
        g.groups = 4


def test_binding_refuses_host_tensors_and_strides():
    """Marshalling: device tensors, contiguous, of the type and size that the call reads."""
    s, g = moe.Shape(4, 64, 64, 8, 2), moe.Gate()
    f, i = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="logits: expected a device tensor"):
        moe.moe_gate_fwd(s, g, f, None, i, torch.zeros(4, 2))
    with pytest.raises(ValueError, match="x: expected a device tensor"):
        moe.moe_norm_fwd(True, 1e-6, torch.zeros(4, 64, dtype=torch.bfloat16), None, None, None, None, None, None, None)
    with pytest.raises(ValueError, match="h: expected rows"):
        moe.moe_norm_bwd(True, f, torch.zeros(()), None, None, None, None, None, None, None, False, None)


@pytest.mark.parametrize("args", ["--groups 3", "--groups 0", "--groups 8 --groups-kept 9", "--groups 8 --groups-kept 0", "--experts 8 --groups 8 --group-best 2",
                                  "--group-best 3", "--experts 8 --groups 8 --groups-kept 1 --top-k 2", "--scale 0 --scores sigmoid", "--scale nan", "--balance-steps -1",
                                  "--balance-rate -1", "--balance-rate inf", "--norm rms --dims 16448x64"])
def test_command_refuses(args, capsys):
    with pytest.raises(SystemExit) as e:
        serve.main(args.split())
    assert e.value.code == 2 and "error: --" in capsys.readouterr().err


def test_served_layer_refuses():
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    args = (z(8, 64), z(8, 64, 64), z(8, 64, 64), z(8, 64, 64), 2)
    for bad in (dict(bias=torch.zeros(8)), dict(gate=moe.Gate(), bias=torch.zeros(7)), dict(norm=(z(63), None, True, 1e-6)), dict(norm=(z(64), z(65), True, 1e-6))):
        with pytest.raises(ValueError):
            serve.ServedLayer(*args, mxfp4=False, **bad)
