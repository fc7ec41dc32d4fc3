"""What stands in front of the experts, as calls of the package's entry points (`own`) and in a plain form of elementary torch operations.

A case is a dict of plain values.  `kind` says which operator one pass goes through:

  gate      router logits to experts and weights.  scores: "softmax" or "sigmoid" over the E experts; the selection goes by score + bias (bias: a
            number per expert; without it by the logits), among the `kept` best of `groups` equal groups of experts (a group's score: the sum of its
            `best` best selection scores), ties to the lowest id; weights: the k scores (without the bias), divided by their sum (renorm), times `scale`;
            Es shared experts more with weight 1.
  gate_bwd  its gradient from that of the weights.  With balance > 0 also the loss  balance E / (k T^2) sum_e n_e sum_t q_te  (n: slots of an
            expert, q: a token's scores divided by their sum) and its gradient.
  norm      layer norm (centre) or RMS norm of rows, with the residual sum in front of it (addend).
  norm_bwd  its gradients: of the rows, with that of the residual sum added (addend), and of the weights.

mask: "experts" (a fifth of them have logits of -1e30), "rows" (one row in 16 is padding, all of its logits are -inf) or "none".  A masked expert
has score 0 and comes after all others; a row that is masked whole gets its lowest ids with weight 0.
"""
import math

import torch

own = False
_MASKED = -1e30
_EPS = 1e-6


def _gate(name, T, E, k, scores, groups=1, kept=1, best=1, bias=False, Es=0, renorm=True, scale=1.0, mask="none"):
    return {"name": name, "kind": "gate", "T": T, "E": E, "k": k, "scores": scores, "groups": groups, "kept": kept, "best": best, "bias": bias, "Es": Es,
            "renorm": renorm, "scale": scale, "mask": mask}


def _gate_bwd(name, *args, balance=0.0, **kw):
    return {**_gate(name, *args, **kw), "kind": "gate_bwd", "balance": balance}


def _norm(name, kind, rows, cols, centre, addend=False, beta=False):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "centre": centre, "addend": addend, "beta": beta}


def listed():
    return [
        # a step of one sequence: nothing but latency
        _gate("gate_one", 1, 64, 6, "softmax", Es=2),
        # a padded prompt of odd length on an odd number of experts, weights as they are
        _gate("gate_odd", 1003, 60, 4, "softmax", groups=6, kept=3, bias=True, renorm=False, Es=1, mask="rows"),
        # many experts of which a fifth are switched off
        _gate("gate_many", 16384, 128, 4, "sigmoid", bias=True, mask="experts"),
        # the largest training batch, experts in groups by device
        _gate("gate_groups", 65536, 256, 8, "sigmoid", groups=8, kept=4, best=2, bias=True, Es=1, scale=2.5),
        # a small batch with the balance loss
        _gate_bwd("gate_bwd_small", 256, 8, 2, "softmax", balance=0.01),
        # the largest batch with the balance loss: every score is needed
        _gate_bwd("gate_bwd_groups", 65536, 256, 8, "sigmoid", groups=8, kept=4, best=2, bias=True, Es=1, scale=2.5, balance=0.001),
        # a step of one sequence, residual sum and norm
        _norm("norm_one", "norm", 1, 4096, False, addend=True),
        # an odd prompt, layer norm with weight and offset
        _norm("norm_odd", "norm", 1003, 1088, True, beta=True),
        # a training batch with the residual sum
        _norm("norm_long", "norm", 16384, 4096, False, addend=True),
        # a small batch: latency, and sums over few rows
        _norm("norm_bwd_small", "norm_bwd", 256, 512, True, addend=True, beta=True),
        # odd sizes
        _norm("norm_bwd_odd", "norm_bwd", 4099, 2056, False),
        # a large batch of wide rows
        _norm("norm_bwd_long", "norm_bwd", 32768, 7168, False, addend=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 65536 tokens or rows, 4 to 1024 experts in up to 16 groups, rows of 64 to 16384 values in multiples of 8."""
    kind = rng.choice(["gate", "gate", "gate_bwd", "norm", "norm_bwd"])
    while True:
        if kind in ("gate", "gate_bwd"):
            T, groups = _log_int(rng, 1, 65536), rng.choice([1, 1, 2, 3, 4, 5, 8, 8, 16])
            size = _log_int(rng, max(2, 4 // groups), 1024 // groups)
            if T * groups * size > 65536 * 256:
                continue
            kept = rng.randint(1, groups)
            k = _log_int(rng, 1, min(16, kept * size))
            args = ("", T, groups * size, k, rng.choice(["softmax", "sigmoid"]))
            kw = dict(groups=groups, kept=kept, best=rng.choice([1, 2]), bias=rng.random() < 0.6, Es=rng.choice([0, 0, 1, 2]), renorm=rng.random() < 0.7,
                      scale=rng.choice([1.0, 1.0, 2.5]), mask=rng.choice(["none", "none", "experts", "rows"]))
            if k == 1 and kind == "gate_bwd":
                kw["renorm"] = False   # (a weight divided by itself has no gradient)
            c = _gate(*args, **kw) if kind == "gate" else _gate_bwd(*args, **kw, balance=rng.choice([0.0, 0.01]))
        else:
            rows, cols = _log_int(rng, 1, 65536), 8 * _log_int(rng, 8, 2048)
            if rows * cols > 32768 * 7168:
                continue
            c = _norm("", kind, rows, cols, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5)
        break
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*size, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.randn(*size, device="cuda", generator=gen).mul_(std).add_(mean).to(dtype)

    st, bf = {"case": dict(case)}, torch.bfloat16
    if case["kind"] in ("gate", "gate_bwd"):
        T, E = case["T"], case["E"]
        st["logits"] = normal(T, E).add_(normal(E, std=0.5))   # (experts differ in popularity)
        if case["mask"] == "experts":
            st["logits"][:, torch.randperm(E, device="cuda", generator=gen)[:E // 5]] = _MASKED
        elif case["mask"] == "rows":
            st["logits"][torch.rand(T, device="cuda", generator=gen) < 1 / 16] = -math.inf
        st["bias"] = normal(E, std=0.05 if case["scores"] == "sigmoid" else 0.2 / E) if case["bias"] else None
        if case["kind"] == "gate_bwd":
            got = _plain_gate(case, st["logits"], st["bias"])
            st.update(got, dtopk_w=normal(*got["topk_w"].shape, std=1 / T),
                      counts=torch.bincount(got["topk_idx"].reshape(-1).long(), minlength=E + case["Es"]).to(torch.int32))
        return st
    rows, cols = case["rows"], case["cols"]
    # a residual stream: channels of different size, a few of them large
    channel = torch.exp(normal(cols, std=0.5))
    channel[torch.rand(cols, device="cuda", generator=gen) < 0.002] *= 20
    st["x"] = normal(rows, cols).mul_(channel).to(bf)
    st["gamma"], st["beta"] = normal(cols, std=0.1, mean=1.0, dtype=bf), normal(cols, std=0.1, dtype=bf) if case["beta"] else None
    st["addend"] = normal(rows, cols, std=0.3 if case["kind"] == "norm" else 1.0, dtype=bf) if case["addend"] else None
    if case["kind"] == "norm_bwd":
        x = st["x"].float()
        mean = x.mean(1, keepdim=True) if case["centre"] else torch.zeros(rows, 1, device="cuda")
        st["mean"] = mean.squeeze(1).contiguous() if case["centre"] else None
        st["rstd"] = (x - mean).square().mean(1).add(_EPS).rsqrt()
        st["dy"] = normal(rows, cols, dtype=bf)
    return st


# ---- one pass --------------------------------------------------------------------------------------------------


def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    kind = case["kind"]
    if kind == "gate":
        return _plain_gate(case, st["logits"], st["bias"])
    if kind == "gate_bwd":
        return _plain_gate_bwd(case, st)
    x = st["x"].float()
    gamma = st["gamma"].float()
    if kind == "norm":
        out = {}
        if case["addend"]:
            out["sum"] = (x + st["addend"].float()).to(torch.bfloat16)
            x = out["sum"].float()
        mean = x.mean(1, keepdim=True) if case["centre"] else 0.0
        rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + _EPS)
        y = (x - mean) * rstd * gamma
        out["y"] = (y + st["beta"].float() if case["beta"] else y).to(torch.bfloat16)
        out["rstd"] = rstd.squeeze(1)
        if case["centre"]:
            out["mean"] = mean.squeeze(1)
        return out
    dy, rstd = st["dy"].float(), st["rstd"].unsqueeze(1)
    xhat = (x - st["mean"].unsqueeze(1) if case["centre"] else x) * rstd
    g = dy * gamma
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if case["centre"]:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd
    if case["addend"]:
        dx = dx + st["addend"].float()
    out = {"dx": dx.to(torch.bfloat16), "dgamma": (dy * xhat).sum(0)}
    if case["beta"]:
        out["dbeta"] = dy.sum(0)
    return out


def _scores(case, logits):
    """fp32 logits -> (64-bit logits, which experts are masked, 64-bit scores): the selection is decided by values that lie next to each other."""
    l = logits.double().clamp(-3.4e38, 3.4e38)
    masked = torch.isnan(logits) | (logits <= _MASKED)
    if case["scores"] == "sigmoid":
        s = 1 / (1 + torch.exp(-l))
    else:
        s = torch.exp(l - l.masked_fill(masked, -math.inf).amax(1, keepdim=True).clamp(min=_MASKED))
        s = s / s.masked_fill(masked, 0.0).sum(1, keepdim=True)
    return l, masked, s.masked_fill(masked, 0.0)


def _plain_gate(case, logits, bias):
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    l, masked, s = _scores(case, logits)
    chosen_by = (l if bias is None else s + bias.double()).masked_fill(masked, -math.inf)
    if G > 1:
        of = (l if bias is None and case["best"] == 1 else s if bias is None else s + bias.double()).masked_fill(masked, -math.inf).view(T, G, E // G)
        best = torch.sort(of, dim=2, descending=True)[0][:, :, :case["best"]]
        dead = torch.isinf(best[:, :, 0])
        group = torch.where(torch.isinf(best), 0.0, best).sum(2).masked_fill(dead, -math.inf)
        order = torch.sort(group, dim=1, descending=True, stable=True)[1]
        keep = torch.zeros(T, G, dtype=torch.bool, device=l.device).scatter_(1, order[:, :case["kept"]], True)
        rank = torch.where(torch.isinf(chosen_by), -1e300, chosen_by)   # (masked ones of a group that stays come before those of one that does not)
        chosen_by = rank.masked_fill(~keep.repeat_interleave(E // G, 1), -math.inf)
    idx = torch.sort(chosen_by, dim=1, descending=True, stable=True)[1][:, :k]
    w = torch.gather(s, 1, idx)
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    w = w * case["scale"]
    shared = torch.arange(E, E + case["Es"], device=l.device).expand(T, case["Es"])
    return {"topk_idx": torch.cat([idx, shared], 1).to(torch.int32), "topk_w": torch.cat([w, torch.ones_like(shared, dtype=w.dtype)], 1).float()}


def _plain_gate_bwd(case, st):
    T, E, k = case["T"], case["E"], case["k"]
    _, _, s = _scores(case, st["logits"])
    s = s.float()
    idx, w, dw = st["topk_idx"][:, :k].long(), st["topk_w"][:, :k], st["dtopk_w"][:, :k]
    inner = (w * dw).sum(1, keepdim=True)
    if case["renorm"]:
        d = w * (dw - inner / case["scale"])
    else:
        d = w * dw
    slope = 1 - s if case["scores"] == "sigmoid" else torch.ones_like(s)
    dlogits = torch.zeros(T, E, device=s.device).scatter_(1, idx, d) * slope
    if case["scores"] == "softmax" and not case["renorm"]:
        dlogits = dlogits - s * inner
    if not case["balance"]:
        return {"dlogits": dlogits}
    total = s.sum(1, keepdim=True)
    q = torch.where(total > 0, s / total, 0.0)
    cost = st["counts"][:E].float() * (case["balance"] * E / (k * float(T) * T))
    mean = (q * cost).sum(1, keepdim=True)
    return {"dlogits": dlogits + q * slope * (cost - mean), "loss": mean.sum()}


def _kept(st, name, make):
    """What a user's program makes once and keeps: buffers, workspaces, the shape."""
    if name not in st:
        st[name] = make()
    return st[name]


def _run_own(case, st):
    import paper_2605_05049_amd as moe
    kind = case["kind"]

    def buffer(name, *size, dtype=torch.float32):
        return _kept(st, name + "_out", lambda: torch.empty(*size, dtype=dtype, device="cuda"))

    if kind in ("gate", "gate_bwd"):
        T, E, Kp = case["T"], case["E"], case["k"] + case["Es"]
        shape = _kept(st, "shape", lambda: moe.Shape(T, 64, 64, E, case["k"], case["Es"], case["renorm"]))
        gate = _kept(st, "gate", lambda: moe.Gate(case["scores"], case["groups"], case["kept"], case["best"], case["scale"]))
        if kind == "gate":
            out = {"topk_idx": buffer("idx", T, Kp, dtype=torch.int32), "topk_w": buffer("w", T, Kp)}
            moe.moe_gate_fwd(shape, gate, st["logits"], st["bias"], out["topk_idx"], out["topk_w"])
            return out
        out, loss, ws = {"dlogits": buffer("dlogits", T, E)}, None, None
        if case["balance"]:
            loss, ws = buffer("loss", 1), _kept(st, "ws", lambda: torch.empty(4096, dtype=torch.uint8, device="cuda"))   # (what the loss needs)
            out["loss"] = loss[0]
        moe.moe_gate_bwd(shape, gate, st["dtopk_w"], st["logits"], st["topk_idx"], st["topk_w"], st["counts"] if case["balance"] else None, case["balance"],
                         out["dlogits"], loss, ws)
        return out
    rows, cols, bf = case["rows"], case["cols"], torch.bfloat16
    if kind == "norm":
        out = {"y": buffer("y", rows, cols, dtype=bf), "rstd": buffer("rstd", rows)}
        if case["addend"]:
            out["sum"] = buffer("sum", rows, cols, dtype=bf)
        if case["centre"]:
            out["mean"] = buffer("mean", rows)
        moe.moe_norm_fwd(case["centre"], _EPS, st["x"], st["addend"], st["gamma"], st["beta"], out.get("sum"), out["y"], out.get("mean"), out["rstd"])
        return out
    out = {"dx": buffer("dx", rows, cols, dtype=bf), "dgamma": buffer("dgamma", cols)}
    if case["beta"]:
        out["dbeta"] = buffer("dbeta", cols)
    ws = _kept(st, "ws", lambda: torch.empty(moe.norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda"))
    moe.moe_norm_bwd(case["centre"], st["dy"], st["x"], st["gamma"], st["mean"], st["rstd"], st["addend"], out["dx"], out["dgamma"], out.get("dbeta"), False, ws)
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------------------


def work(case):
    if case["kind"] in ("gate", "gate_bwd"):
        T, E, Kp = case["T"], case["E"], case["k"] + case["Es"]
        if case["kind"] == "gate":
            return {"bytes": 4.0 * T * E + 8.0 * T * Kp + 4.0 * E * case["bias"], "flops": 4.0 * T * E}
        # the logits of all experts where their scores count, else of the chosen ones
        dense = case["balance"] > 0 or (case["scores"] == "softmax" and not case["renorm"])
        read = E if dense else case["k"] if case["scores"] == "sigmoid" else 0
        return {"bytes": 4.0 * T * (E + read) + 12.0 * T * case["k"] + (4.0 * E if case["balance"] else 0.0), "flops": (10.0 if dense else 1.0) * T * E}
    n = float(case["rows"] * case["cols"])
    extra = (4 if case["kind"] == "norm" else 2) * case["addend"]
    if case["kind"] == "norm":
        return {"bytes": (4 + extra) * n + 4.0 * case["rows"] * (1 + case["centre"]) + 2.0 * case["cols"] * (1 + case["beta"]), "flops": 6 * n}
    return {"bytes": (6 + extra) * n + 4.0 * case["rows"] * (1 + case["centre"]) + case["cols"] * (6.0 + 4 * case["beta"]), "flops": 12 * n}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------


def _exact_scores(case, logits):
    dead = torch.isnan(logits) | (logits <= _MASKED)
    l = logits.double()
    s = torch.sigmoid(l) if case["scores"] == "sigmoid" else torch.softmax(torch.where(dead, -math.inf, l), 1)
    return torch.where(dead, 0.0, torch.nan_to_num(s))   # (a row without experts: 0 / 0)


def _exact_weights(case, s, idx):
    w = s.gather(1, idx)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return w * case["scale"]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("gate", "gate_bwd"):
        T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
        logits = st["logits"]
        if kind == "gate":
            s = _exact_scores(case, logits)
            dead = torch.isnan(logits) | (logits <= _MASKED)
            c = torch.where(dead, -100.0, s if st["bias"] is None else s + st["bias"].double())
            of = torch.topk(c.view(T, G, -1), case["best"], dim=2)[0]
            of = torch.where(of[:, :, :1] < -50, -1000.0, torch.where(of < -50, 0.0, of)).sum(2)
            worst = torch.topk(of, case["kept"], dim=1)[0][:, -1:]     # (groups without a living expert: which of them stay does not change a weight)
            c = torch.where((of >= worst).unsqueeze(2), c.view(T, G, -1), -1e4).view(T, E)
            w = _exact_weights(case, s, torch.topk(c, k, dim=1)[1])
            return {"topk_idx": None, "topk_w": torch.cat([w, torch.ones(T, case["Es"], dtype=w.dtype, device=w.device)], 1)}
        with torch.enable_grad():   # by differentiating the definition
            l = logits.double().requires_grad_()
            fine = torch.where(torch.isnan(logits) | (logits <= _MASKED), torch.full_like(l, _MASKED), l)
            alive = logits > _MASKED
            none = ~alive.any(1, keepdim=True)
            s = (torch.sigmoid(fine) if case["scores"] == "sigmoid" else torch.softmax(fine, 1)) * alive
            idx = st["topk_idx"][:, :k].long()
            total = (_exact_weights(case, s, idx) * st["dtopk_w"][:, :k].double()).sum()
            out = {}
            if case["balance"]:
                q = s / torch.where(none, 1.0, s.sum(1, keepdim=True))
                loss = case["balance"] * E / k * (st["counts"][:E].double() / T * (q.sum(0) / T)).sum()
                out["loss"] = loss.detach()
                total = total + loss
            out["dlogits"] = torch.autograd.grad(total, l)[0]
        return out
    bf = torch.bfloat16
    gamma = st["gamma"].double()
    beta = st["beta"].double() if case["beta"] else torch.zeros_like(gamma)
    if kind == "norm":
        h = (st["x"].float() + st["addend"].float()).to(bf) if case["addend"] else st["x"]   # (the norm is that of the sum as it is stored)
        h = h.double()
        mean = h.mean(1) if case["centre"] else torch.zeros_like(h[:, 0])
        h -= mean.unsqueeze(1)
        rstd = (h.pow(2).mean(1) + _EPS).pow(-0.5)
        out = {"y": torch.addcmul(beta, h.mul_(rstd.unsqueeze(1)), gamma), "rstd": rstd}
        if case["centre"]:
            out["mean"] = mean
        if case["addend"]:
            out["sum"] = st["x"].double() + st["addend"].double()
        return out
    out = {"dx": torch.empty(case["rows"], case["cols"], dtype=torch.float64, device="cuda")}
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(gamma)
    for at in range(0, case["rows"], 4096):   # by differentiating the definition, some rows at a time
        part = slice(at, at + 4096)
        with torch.enable_grad():
            x, a, b = st["x"][part].double().requires_grad_(), gamma.clone().requires_grad_(), beta.clone().requires_grad_()
            h = x - x.mean(1, keepdim=True) if case["centre"] else x
            y = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + _EPS) * a + b
            dx, da, db = torch.autograd.grad(y, (x, a, b), st["dy"][part].double())
        out["dx"][part] = dx + st["addend"][part].double() if case["addend"] else dx
        dgamma += da
        dbeta += db
    out["dgamma"] = dgamma
    if case["beta"]:
        out["dbeta"] = dbeta
    return out
