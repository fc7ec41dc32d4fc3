"""Buffer set and call order of one MoE expert layer step.  Torch is used for device memory only: every
computation is one of the C-ABI entry points, called in the order of the per-layer flow (routing -> pack ->
experts -> unpack/combine, then the reverse for backward)."""
from __future__ import annotations

import contextlib
import math

from . import binding as B


def on_stream(stream):
    """Within it, memory is allocated for work on `stream`: another stream's pool hands out what its own work may still be reading."""
    if stream is None:
        return contextlib.nullcontext()
    import torch
    return torch.cuda.stream(stream)


class MoeLayerBuffers:
    """All device buffers one forward+backward of a layer touches, allocated once.  `empty(*size, dtype=...)` allocates them (all but out).  Without
    `with_saved` nothing is kept for a backward (save_g and save_u are None), and of `mxfp4` the workspace is that of layer_mxfp4_forward."""

    def __init__(self, shape, device="cuda", with_backward=True, with_router=True, empty=None, with_saved=True, mxfp4=False):
        import torch
        s = B.Shape.of(shape)
        self.shape = s
        dev = torch.device(device)
        bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
        N, T, d, f, Et, Kp = s.N, s.T, s.d_model, s.d_ffn, s.E_total, s.K_slots
        e = empty or (lambda *sz, dtype: torch.empty(*sz, dtype=dtype, device=dev))
        self.topk_idx = e(T, Kp, dtype=i32)
        self.topk_w = e(T, Kp, dtype=f32)
        self.probs = e(T, s.E, dtype=f32) if with_router else None
        self.counts = e(Et, dtype=i32)
        self.offsets = e(Et + 1, dtype=i32)
        self.row_of_slot = e(N, dtype=i32)
        self.slot_of_row = e(N, dtype=i32)
        self.x_perm = e(N, d, dtype=bf)
        self.save_g = e(N, f, dtype=bf) if with_saved else None
        self.save_u = e(N, f, dtype=bf) if with_saved else None
        self.y_perm = e(N, d, dtype=bf)
        self.out = torch.empty(T, d, dtype=bf, device=dev)
        self.ws = e(max((B.mxfp4_workspace_bytes if mxfp4 else B.workspace_bytes)(s), 256), dtype=torch.uint8)
        if with_backward:
            self.dy_perm = e(N, d, dtype=bf)
            self.dtopk_w = e(T, Kp, dtype=f32)
            self.dx_perm = e(N, d, dtype=bf)
            self.dx = e(T, d, dtype=bf)
            self.dw_gate = e(Et, d, f, dtype=f32)
            self.dw_up = e(Et, d, f, dtype=f32)
            self.dw_down = e(Et, f, d, dtype=f32)
            self.dlogits = e(T, s.E, dtype=f32) if with_router else None
        # the layer closed from x (router weight given): logits, the router's term of dx, the router weight gradient
        self.logits = e(T, s.E, dtype=f32) if with_router else None
        if with_backward and with_router:
            self.dx_router = e(T, d, dtype=bf)
            self.dw_router = e(s.E, d, dtype=f32)
            self.balance_loss = e(1, dtype=f32)
            self.routed_by = self.logits   # what the last forward call routed by, for the backward of a gate


class _Carved:
    """Tensors next to each other in a block of bytes; without a block, how many they would take (`at`)."""

    def __init__(self, block=None):
        self.block, self.at = block, 0

    def __call__(self, *size, dtype):
        at, n = self.at, math.prod(size) * dtype.itemsize
        self.at += -(-n // 256) * 256
        return None if self.block is None else self.block[at:at + n].view(dtype).view(size)


class PromptMemory:
    """The memory of forward calls with any number of tokens, one after another: a block that the longest so far needs.  Each call's `out` is its
    own; the other buffers of a shape are good until those of another one are asked for.  `mxfp4`: of layer_mxfp4_forward."""

    _VIEWS = 256   # shapes whose buffers in the block are kept as they are (tensors without memory of their own)

    def __init__(self, device="cuda", mxfp4=False):
        self._kind = {"with_backward": False, "with_saved": False, "mxfp4": mxfp4}
        self.device, self.block, self._views, self._latest = device, None, {}, None
        self.streams = set()   # that used the block

    def buffers(self, shape) -> MoeLayerBuffers:
        s = B.Shape.of(shape)
        key = (s.T, s.d_model, s.d_ffn, s.E, s.k, s.E_shared, s.renorm)
        buf = self._views.get(key)
        if buf is not None and buf is self._latest:
            return buf
        import torch
        if buf is None:
            need = _Carved()
            MoeLayerBuffers(s, self.device, empty=need, **self._kind)
            if self.block is None or self.block.numel() < need.at:
                self._views, self._latest, self.block, self.streams = {}, None, None, set()   # (the old block goes first)
                self.block = torch.empty(need.at, dtype=torch.uint8, device=self.device)
            elif len(self._views) >= self._VIEWS:
                self._views = {}
            buf = self._views[key] = MoeLayerBuffers(s, self.device, empty=_Carved(self.block), **self._kind)
        if buf is not self._latest:
            if self._latest is not None:
                self._latest.out = None
            if buf.out is None:
                buf.out = torch.empty(s.T, s.d_model, dtype=torch.bfloat16, device=self.device)
            self._latest = buf
        return buf


def _route(buf, x, logits, w_router, gate, bias, stream):
    """topk_idx and topk_w of a layer's buffers, from logits or from x (buf.logits = x W_r^T); neither given: they are there already."""
    s = buf.shape
    if gate is None and bias is not None:
        raise ValueError("bias: goes with a gate")
    if gate is not None and logits is not None and w_router is not None:   # (a backward call with both would not know which)
        raise ValueError("gate: it routes by logits or by those of w_router, not by both")
    if gate is not None and w_router is not None:
        B.moe_router_gate_fwd(s, gate, x, w_router, bias, buf.logits, buf.topk_idx, buf.topk_w, buf.ws, stream)
    elif gate is not None and logits is not None:
        B.moe_gate_fwd(s, gate, logits, bias, buf.topk_idx, buf.topk_w, stream)
    elif gate is not None:
        raise ValueError("gate: without logits and w_router there is nothing to route by")
    elif w_router is not None:
        B.moe_router_route_fwd(s, x, w_router, buf.logits, buf.topk_idx, buf.topk_w, buf.probs, buf.ws, stream)
    elif logits is not None:
        B.moe_route_topk(s, logits, buf.topk_idx, buf.topk_w, buf.probs, stream)


def layer_forward(buf: MoeLayerBuffers, x, w_gate, w_up, w_down, logits=None, w_router=None, stream=None, gate=None, bias=None):
    """routing (skipped when logits is None: buf.topk_idx / buf.topk_w were filled by the caller, as for an
    expert-parallel shard) -> permute -> grouped FFN -> combine.  With `w_router` the logits are computed first
    (buf.logits = x W_r^T).  `gate` (a binding.Gate) routes by its scores and groups, by `logits` or by those of `w_router`, `bias` [E] fp32 shifts
    its choice.  Returns buf.out."""
    s = buf.shape
    _route(buf, x, logits, w_router, gate, bias, stream)
    if hasattr(buf, "routed_by"):
        buf.routed_by = buf.logits if logits is None or w_router is not None else logits
    B.moe_permute(s, x, buf.topk_idx, buf.x_perm, buf.counts, buf.offsets, buf.row_of_slot, buf.slot_of_row, buf.ws, stream)
    B.moe_grouped_ffn_fwd(s, buf.x_perm, buf.offsets, w_gate, w_up, w_down, buf.y_perm, buf.save_g, buf.save_u, buf.ws, stream)
    B.moe_unpermute_combine(s, buf.y_perm, buf.row_of_slot, buf.topk_w, buf.out, stream)
    return buf.out


def layer_backward(buf: MoeLayerBuffers, dout, w_gate, w_up, w_down, accumulate=False, with_router=True, x=None,
                   w_router=None, stream=None, gate=None, logits=None, balance=0.0):
    """combine_bwd and route_bwd (one launch) -> grouped FFN bwd -> permute_bwd.  Results land in buf.dx, buf.dw_*,
    buf.dtopk_w, buf.dlogits.  With `x` and `w_router` the layer is closed from x: router_bwd comes with the
    experts' backward, buf.dx then holds the expert-path term plus the router's term, and buf.dw_router is filled.
    `gate`: that of the forward call; its logits are taken (buf.routed_by: those given to it, or buf.logits) unless others are given.  With `balance` the gradient of the balance loss is part of
    buf.dlogits (by buf.counts), its value in buf.balance_loss."""
    s = buf.shape
    gated = with_router and buf.dlogits is not None
    if gate is None and balance:
        raise ValueError("balance: goes with a gate")
    if gate is not None:
        if buf.dlogits is None:
            raise ValueError("gate: these buffers have none for a router")
        B.moe_unpermute_combine_bwd(s, dout, buf.y_perm, buf.row_of_slot, buf.topk_w, buf.dy_perm, buf.dtopk_w, stream)
        B.moe_gate_bwd(s, gate, buf.dtopk_w, buf.routed_by if logits is None else logits, buf.topk_idx, buf.topk_w, buf.counts if balance else None, balance,
                       buf.dlogits, buf.balance_loss if balance else None, buf.ws, stream)
    elif gated or w_router is not None:   # (a token's dlogits need no more than its dtopk_w: made with it, not after the experts' backward)
        B.moe_unpermute_combine_route_bwd(s, dout, buf.y_perm, buf.row_of_slot, buf.topk_idx, buf.topk_w, buf.probs, buf.dy_perm, buf.dtopk_w,
                                          buf.dlogits, stream)
    else:
        B.moe_unpermute_combine_bwd(s, dout, buf.y_perm, buf.row_of_slot, buf.topk_w, buf.dy_perm, buf.dtopk_w, stream)
    ffn = (buf.dy_perm, buf.x_perm, buf.offsets, w_gate, w_up, w_down, buf.save_g, buf.save_u, buf.dx_perm, buf.dw_gate, buf.dw_up, buf.dw_down)
    if w_router is not None:
        B.moe_grouped_ffn_router_bwd(s, *ffn, x, w_router, buf.dlogits, buf.dx_router, buf.dw_router, accumulate, buf.ws, stream)
        B.moe_permute_bwd_add(s, buf.dx_perm, buf.row_of_slot, buf.dx_router, buf.dx, stream)
    else:
        B.moe_grouped_ffn_bwd(s, *ffn, accumulate, buf.ws, stream)
        B.moe_permute_bwd(s, buf.dx_perm, buf.row_of_slot, buf.dx, stream)


class CapturedLayerStep:
    """One forward+backward of a layer recorded into a HIP graph and replayed with a single launch.

    Every node of the graph is one of the library's kernels: the entry points allocate nothing, never synchronise
    the host, take the ragged counts from device memory and clear their own counters with kernels (no memset
    nodes), so a whole step can be captured.  torch.cuda.CUDAGraph drives the capture.  The tensors passed in are the
    graph's static inputs: refill them in place (`x.copy_(...)`) and call `replay()`; results land in `buf` as
    after `layer_forward` + `layer_backward`."""

    def __init__(self, buf: MoeLayerBuffers, x, dout, w_gate, w_up, w_down, logits=None, w_router=None,
                 accumulate=False, with_router=True, warmup=2, gate=None, bias=None, balance=0.0):
        import torch
        self.buf = buf
        self._args = (x, dout, w_gate, w_up, w_down, logits, w_router, accumulate, with_router)
        self._gate = (gate, bias, balance)
        side = torch.cuda.Stream()  # default priority
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(warmup):
                self._step()
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._step()

    def _step(self):
        x, dout, w_gate, w_up, w_down, logits, w_router, accumulate, with_router = self._args
        gate, bias, balance = self._gate
        layer_forward(self.buf, x, w_gate, w_up, w_down, logits=logits, w_router=w_router, gate=gate, bias=bias)
        layer_backward(self.buf, dout, w_gate, w_up, w_down, accumulate=accumulate, with_router=with_router,
                       x=x if w_router is not None else None, w_router=w_router, gate=gate, logits=logits, balance=balance)

    def replay(self):
        self.graph.replay()


class MoeBlockBuffers:
    """What a layer with the residual sum and the norm in front of it touches: `layer`, the layer's buffers; h, the residual sum; y, its norm; mean
    (centred) and rstd; with a backward dh, dgamma, dbeta.  centre: layer norm, else RMS norm."""

    def __init__(self, shape, centre=False, eps=1e-6, device="cuda", with_backward=True):
        import torch
        s = B.Shape.of(shape)
        T, d, dev = s.T, s.d_model, torch.device(device)
        if not B.norm_workspace_bytes(T, d):
            raise ValueError(f"d_model {d}: the norm takes up to {B.NORM_COLS_MAX}")
        self.shape, self.centre, self.eps = s, bool(centre), float(eps)
        self.layer = MoeLayerBuffers(s, device, with_backward=with_backward, with_saved=with_backward)
        e = lambda *size, dtype=torch.bfloat16: torch.empty(*size, dtype=dtype, device=dev)  # noqa: E731
        self.h, self.y = e(T, d), e(T, d)
        self.mean, self.rstd = e(T, dtype=torch.float32) if centre else None, e(T, dtype=torch.float32)
        if with_backward:
            self.dh, self.dgamma, self.dbeta = e(T, d), e(d, dtype=torch.float32), e(d, dtype=torch.float32)
            self.norm_ws = e(B.norm_workspace_bytes(T, d), dtype=torch.uint8)


def block_forward(buf: MoeBlockBuffers, x, addend, gamma, beta, w_gate, w_up, w_down, w_router, gate=None, bias=None, stream=None):
    """h = x + addend (without an addend h = x), then layer(norm(h)).  addend: what the block before added to the residual stream x; gamma, beta may be
    None.  Returns (h, out): the residual stream and what this layer adds to it, to be summed by the next block."""
    h = x if addend is None else buf.h
    B.moe_norm_fwd(buf.centre, buf.eps, x, addend, gamma, beta, None if addend is None else h, buf.y, buf.mean, buf.rstd, stream)
    return h, layer_forward(buf.layer, buf.y, w_gate, w_up, w_down, w_router=w_router, stream=stream, gate=gate, bias=bias)


def block_backward(buf: MoeBlockBuffers, h, dh, dout, gamma, w_gate, w_up, w_down, w_router, accumulate=False, gate=None, balance=0.0, stream=None,
                   with_beta=True):
    """The backward of block_forward: h as it returned it, dh the gradient that reaches h past this block (may be None), dout that of out.  buf.dh is
    the gradient of x and of addend alike; buf.dgamma (unless gamma is None) and buf.dbeta (unless with_beta is false) those of the norm's weights, and
    the layer's are in buf.layer."""
    layer_backward(buf.layer, dout, w_gate, w_up, w_down, accumulate=accumulate, x=buf.y, w_router=w_router, stream=stream, gate=gate, balance=balance)
    B.moe_norm_bwd(buf.centre, buf.layer.dx, h, gamma, buf.mean, buf.rstd, dh, buf.dh, None if gamma is None else buf.dgamma,
                   buf.dbeta if with_beta else None, accumulate, buf.norm_ws, stream)


class FewTokenBuffers:
    """Outputs and workspace of the layer for a few tokens (at most binding.FEW_TOKENS_MAX).  with_gate: and the logits of a gate of its own."""

    def __init__(self, shape, device="cuda", with_gate=False):
        import torch
        s = B.Shape.of(shape)
        nbytes = B.layer_few_workspace_bytes(s)
        if nbytes == 0:
            raise ValueError(f"the layer for a few tokens takes at most {B.FEW_TOKENS_MAX} tokens of a valid shape")
        self.shape = s
        dev = torch.device(device)
        self.topk_idx = torch.empty(s.T, s.K_slots, dtype=torch.int32, device=dev)
        self.topk_w = torch.empty(s.T, s.K_slots, dtype=torch.float32, device=dev)
        self.out = torch.empty(s.T, s.d_model, dtype=torch.bfloat16, device=dev)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        self.logits = torch.empty(s.T, s.E, dtype=torch.float32, device=dev) if with_gate else None
        self.gate_ws = torch.empty(max(B.mxfp4_workspace_bytes(s), 256), dtype=torch.uint8, device=dev) if with_gate else None
        self.streams = set()   # that used them, if the user keeps account


def layer_few_forward(buf: FewTokenBuffers, x, weights, w_router=None, stream=None, gate=None, bias=None):
    """The whole layer for a few tokens.  weights: (w_gate, w_up, w_down) in bf16, or what quantize_experts returned.  Without `w_router`
    buf.topk_idx / buf.topk_w were filled by the caller, as for an expert-parallel shard.  `gate`, `bias`: as in layer_forward (buffers with_gate).
    Returns buf.out."""
    if gate is not None:
        if w_router is None or buf.logits is None:
            raise ValueError("gate: needs w_router, and buffers with_gate")
        B.moe_router_gate_fwd(buf.shape, gate, x, w_router, bias, buf.logits, buf.topk_idx, buf.topk_w, buf.gate_ws, stream)
        w_router = None
    elif bias is not None:
        raise ValueError("bias: goes with a gate")
    fn = B.moe_layer_few_fwd if len(weights) == 3 else B.moe_layer_few_mxfp4_fwd
    fn(buf.shape, x, w_router, *weights, buf.out, buf.topk_idx, buf.topk_w, buf.ws, stream)
    return buf.out


def quantize_experts(w_gate, w_up, w_down, stream=None):
    """The experts' weights in microscaled 4-bit floating point, blocks along each contraction: (q, scales) of W_gate, W_up [E', f, d / 2]
    and W_down [E', d, f / 2].  Once, when a model is loaded."""
    import torch
    got = []
    for w in (w_gate, w_up, w_down):
        E, K, C = w.shape
        with on_stream(stream):
            q = torch.empty(E, C, K // 2, dtype=torch.uint8, device=w.device)
            scales = torch.empty(E, C, K // 32, dtype=torch.uint8, device=w.device)
        B.moe_mxfp4_quantize_t(w, q, scales, stream)
        if stream is not None:
            w.record_stream(stream)   # (the caller may drop it now)
        got += [q, scales]
    return tuple(got)


def layer_mxfp4_forward(buf: MoeLayerBuffers, x, weights, logits=None, w_router=None, stream=None, gate=None, bias=None):
    """layer_forward on weights that quantize_experts returned (a prompt; nothing is kept for a backward pass).  Returns buf.out."""
    s = buf.shape
    _route(buf, x, logits, w_router, gate, bias, stream)
    B.moe_permute(s, x, buf.topk_idx, buf.x_perm, buf.counts, buf.offsets, buf.row_of_slot, buf.slot_of_row, buf.ws, stream)
    B.moe_mxfp4_grouped_ffn_fwd(s, buf.x_perm, buf.offsets, *weights, buf.y_perm, buf.ws, stream)
    B.moe_unpermute_combine(s, buf.y_perm, buf.row_of_slot, buf.topk_w, buf.out, stream)
    return buf.out
