"""Answering with one MoE layer: the experts' weights are quantised to microscaled 4-bit floating point when the layer is loaded, a prompt goes
through the grouped 4-bit products, and the tokens that follow go through the layer for a few tokens.  The grouped products quantise a prompt's rows
and hidden activations to 4 bits, too; the layer for a few tokens (at most 64) keeps the rows in bf16 and 16 significand bits of the hidden activations.

    python -m paper_2605_05049_amd.serve --dims 2048x1408 --experts 64 --top-k 6 --shared 2 --prompt 4096 --batch 1 --steps 64

prints one JSON line: what the weights take, the time of the prompt and of a step (its launches replayed as a graph), and how far the answers
are from those of the bf16 weights."""
import argparse
import json
import sys

from . import binding as B
from .layer import FewTokenBuffers, MoeLayerBuffers, PromptMemory, layer_few_forward, layer_forward, layer_mxfp4_forward, on_stream, quantize_experts


class ServedLayer:
    """A layer that only answers: `layer(x)` for x [T, d_model] bf16, any T.  At most FEW_TOKENS_MAX tokens are answered by layer_few_forward,
    more by the grouped products.  `mxfp4`: the experts' weights are quantised here, and the bf16 ones are not kept; and a call with more than a few tokens
    quantises its rows and hidden activations to 4 bits on the way (its answers are 30 % off those of bf16, of random weights and rows, where a call
    with a few tokens, whose rows stay bf16, is 20 % off).  Without it everything is bf16.

    The buffers of a few tokens are made for their count at its first call and kept; what a call returns is theirs and is overwritten by the next
    call with as many tokens.  Longer calls share the memory of the longest so far, and each returns a tensor of its own.  Memory that a captured
    call uses stays as long as the layer.  Calls on one stream at a time; the memory is freed for others when all streams that had calls are past
    them.

    `gate`, `bias` [E] fp32: routing by the gate's scores, bias and groups.  `norm`: (gamma, beta, centre, eps) of the norm in front of the layer (gamma
    [d_model], beta [d_model] or None, bf16); it is applied by `block`, not by a call."""

    def __init__(self, w_router, w_gate, w_up, w_down, top_k, n_shared=0, renorm=1, mxfp4=True, stream=None, gate=None, bias=None, norm=None):
        E, d = w_router.shape
        n, f = E + n_shared, w_gate.shape[-1]
        if gate is None and bias is not None:
            raise ValueError("bias: goes with a gate")
        if bias is not None and tuple(bias.shape) != (E,):
            raise ValueError(f"bias {tuple(bias.shape)}: expected {(E,)}")
        for name, w in (("gamma", norm[0]), ("beta", norm[1])) if norm is not None else ():
            if w is not None and tuple(w.shape) != (d,):
                raise ValueError(f"{name} {tuple(w.shape)}: expected {(d,)}")
        if norm is not None and d > B.NORM_COLS_MAX:
            raise ValueError(f"d_model {d}: the norm takes up to {B.NORM_COLS_MAX}")
        for name, w, want in (("w_gate", w_gate, (n, d, f)), ("w_up", w_up, (n, d, f)), ("w_down", w_down, (n, f, d))):
            if tuple(w.shape) != want:
                raise ValueError(f"{name} {tuple(w.shape)}: expected {want}")
        self.w_router, self.mxfp4 = w_router, mxfp4
        self.gate, self.bias, self.norm = gate, bias, norm
        self.weights = quantize_experts(w_gate, w_up, w_down, stream) if mxfp4 else (w_gate, w_up, w_down)
        self._fields = (d, f, E, top_k, n_shared, renorm)
        self._few, self._prompts, self._captured = {}, PromptMemory(w_router.device, mxfp4), []
        self._streams = set()   # that had calls

    def buffers(self, T):
        """The buffers of calls with T tokens (topk_idx, topk_w, out, ...); of more than a few tokens good until a call with another number of them."""
        buf = self._few.get(T)
        if buf is None:
            s = B.Shape(T, *self._fields)
            if T > B.FEW_TOKENS_MAX or B.layer_few_workspace_bytes(s) == 0:
                return self._prompts.buffers(s)
            buf = self._few[T] = FewTokenBuffers(s, self.w_router.device, with_gate=self.gate is not None)
        return buf

    def __call__(self, x, stream=None):
        if x.dim() != 2 or x.shape[1] != self._fields[0]:
            raise ValueError(f"x {tuple(x.shape)}: expected [T, {self._fields[0]}]")
        import torch
        with on_stream(stream):
            buf = self.buffers(x.shape[0])
            if isinstance(buf, FewTokenBuffers):
                out = layer_few_forward(buf, x, self.weights, w_router=self.w_router, gate=self.gate, bias=self.bias)
                self._used(buf.streams, vars(buf).values())
                return out
            buf.out = torch.empty_like(buf.out)
            if self.mxfp4:
                out = layer_mxfp4_forward(buf, x, self.weights, w_router=self.w_router, gate=self.gate, bias=self.bias)
            else:
                out = layer_forward(buf, x, *self.weights, w_router=self.w_router, gate=self.gate, bias=self.bias)
            block = self._prompts.block
            self._used(self._prompts.streams, (block,))
            if torch.cuda.is_current_stream_capturing() and not any(b is block for b in self._captured):
                self._captured.append(block)
            return out

    def block(self, x, addend=None, stream=None):
        """The residual sum h = x + addend (h = x without an addend) and layer(norm(h)): returns both, h a tensor of its own (or x itself)."""
        if self.norm is None:
            raise ValueError("a layer without a norm has no block")
        for name, t in (("x", x), ("addend", addend)):
            if t is not None and (t.dim() != 2 or t.shape[1] != self._fields[0] or t.shape != x.shape):
                raise ValueError(f"{name} {tuple(t.shape)}: expected [T, {self._fields[0]}], as x")
        with on_stream(stream):
            h, y = self._normed(x, addend)
            return h, self(y)

    def _normed(self, x, addend=None):
        """h = x + addend (x itself without an addend) and its norm."""
        import torch
        gamma, beta, centre, eps = self.norm
        y = torch.empty_like(x)
        h = x if addend is None else torch.empty_like(x)
        B.moe_norm_fwd(centre, eps, x, addend, gamma, beta, None if addend is None else h, y, None, None)
        return h, y

    def _used(self, streams, tensors):
        """What the call used, these tensors and the weights, is not to be handed out again before the current stream is past it.  (Once per stream: the
        allocator waits for what a stream has enqueued by the time the memory is freed.)"""
        import torch
        handle = B._stream(None)
        if handle in streams and handle in self._streams:
            return
        for seen, what in ((self._streams, (self.w_router, self.bias, *(self.norm or ())[:2], *self.weights)), (streams, tensors)):
            if handle not in seen:
                seen.add(handle)
                for t in what:
                    if isinstance(t, torch.Tensor):
                        t.record_stream(torch.cuda.current_stream())


def _next(x, y):
    """Inputs of the next step: a residual sum, normalised."""
    h = x.float() + y.float()
    return (h * h.square().mean(-1, keepdim=True).add(1e-6).rsqrt()).to(x.dtype)


def answer(layer, prompt, batch, steps):
    """The layer over the prompt, then `steps` steps of the prompt's last `batch` rows; (answers of the prompt, of every step).  With a norm the rows are the
    residual stream, to which every step adds its answers."""
    import torch
    if layer.norm is not None:
        h, y = layer.block(prompt)
        first, h, y, rows = y.clone(), h[-batch:].contiguous(), y[-batch:].clone(), []
        for _ in range(steps):
            h, y = layer.block(h, y)
            y = y.clone()
            rows.append(y)
        return first, torch.stack(rows)
    first = layer(prompt).clone()
    x, rows = _next(prompt[-batch:], first[-batch:]), []
    for _ in range(steps):
        y = layer(x)
        rows.append(y.clone())
        x = _next(x, y)
    return first, torch.stack(rows)


def _ms(fn, repeats):
    import torch
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    fn()
    start.record()
    for _ in range(repeats):
        fn()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) / repeats


def balance(layer, x, steps, rate):
    """`steps` steps of the layer's bias on the loads of x (of its norm, if the layer has one); the largest load over the mean, before and after."""
    if layer.norm is not None:
        _, x = layer._normed(x)
    E, loads = layer.w_router.shape[0], []
    s = B.Shape(x.shape[0], *layer._fields)
    buf = MoeLayerBuffers(s, layer.w_router.device, with_backward=False, with_saved=False)
    for i in range(steps + 1):
        B.moe_router_gate_fwd(s, layer.gate, x, layer.w_router, layer.bias, buf.logits, buf.topk_idx, buf.topk_w, buf.ws)
        B.moe_permute(s, None, buf.topk_idx, None, buf.counts, buf.offsets, buf.row_of_slot, buf.slot_of_row, buf.ws)
        if i in (0, steps):
            loads.append((buf.counts[:E].max() / buf.counts[:E].double().mean()).item())
        if i < steps:
            B.moe_gate_bias_step(s, buf.counts, rate, layer.bias)
    return loads[0], loads[-1]


def run(d, f, experts, top_k, shared, prompt, batch, steps, seed=0, gate=None, norm=None, balance_steps=0, balance_rate=0.002):
    """norm: "rms" or "layer", in front of the layer: then prompt and steps go through `block`.  balance_steps: the gate's bias begins at 0 and takes that
    many steps on the prompt's loads."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std: (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    n = experts + shared
    weights = [torch.stack([normal(*s, std=std) for _ in range(n)]) for s, std in (((d, f), d ** -0.5), ((d, f), d ** -0.5), ((f, d), f ** -0.5))]
    w_router, x = normal(experts, d, std=2 * d ** -0.5), normal(prompt, d, std=1.0)
    front = {}
    if gate is not None:
        front["gate"] = gate
        front["bias"] = torch.zeros(experts, device="cuda") if balance_steps else None
    if norm is not None:
        front["norm"] = (torch.ones(d, dtype=torch.bfloat16, device="cuda"), None, norm == "layer", 1e-6)
    full = ServedLayer(w_router, *weights, top_k, shared, mxfp4=False, **front)
    layer = ServedLayer(w_router, *weights, top_k, shared, **front)
    loads = balance(layer, x, balance_steps, balance_rate) if balance_steps else None
    through = lambda served, *rows: served(*rows) if norm is None else served.block(*rows)[1]  # noqa: E731
    got = through(layer, x).clone()
    ref = through(full, x).float()
    answer(layer, x, batch, steps)
    # a step's rows: the prompt's last ones; with a norm they are the residual stream, to which the prompt's answers are added
    static = [x[-batch:].clone()] + ([] if norm is None else [got[-batch:].clone()])
    got = got.float()
    through(layer, *static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step = through(layer, *static)
    step_ref = through(full, *static).float()
    graph.replay()
    step = step.float()
    off = lambda a, b: round(((a - b).norm() / b.norm()).item(), 4)  # noqa: E731
    return {"d_model": d, "d_ffn": f, "experts": experts, "shared": shared, "top_k": top_k, "prompt": prompt, "batch": batch,
            "weights_GB": round(sum(w.numel() * w.element_size() for w in layer.weights) / 1e9, 3),
            "bf16_weights_GB": round(sum(w.numel() * w.element_size() for w in weights) / 1e9, 3),
            "prompt_ms": round(_ms(lambda: through(layer, x), 5), 4), "bf16_prompt_ms": round(_ms(lambda: through(full, x), 5), 4),
            "step_us": round(1e3 * _ms(graph.replay, max(1, steps)), 2), "off_prompt": off(got, ref), "off_step": off(step, step_ref),
            **({"load_before": round(loads[0], 3), "load_after": round(loads[1], 3)} if loads else {})}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--dims", default="2048x1408", help="d_model x d_ffn")
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--top-k", type=int, default=6)
    ap.add_argument("--shared", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=4096, help="tokens")
    ap.add_argument("--batch", type=int, default=1, help="tokens of a step")
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--scores", choices=("softmax", "sigmoid"), default="softmax", help="of the router")
    ap.add_argument("--groups", type=int, default=1, help="of experts")
    ap.add_argument("--groups-kept", type=int, default=None, help="for a token (all)")
    ap.add_argument("--group-best", type=int, default=1, help="scores that are summed to a group's: 1 or 2")
    ap.add_argument("--scale", type=float, default=1.0, help="on the weights")
    ap.add_argument("--norm", choices=("rms", "layer"), default=None, help="in front of the layer")
    ap.add_argument("--balance-steps", type=int, default=0, help="of a bias that evens the experts' loads, on the prompt")
    ap.add_argument("--balance-rate", type=float, default=0.002)
    args = ap.parse_args(argv)
    import torch
    B.load_library()
    if not 1 <= args.batch <= args.prompt:
        ap.error("--batch is between 1 and --prompt")
    if args.steps < 1:
        ap.error("--steps is at least 1")
    try:
        d, f = (int(v) for v in args.dims.lower().split("x"))
    except ValueError:
        ap.error("--dims is two numbers, as 2048x1408")
    if B.workspace_bytes(B.Shape(args.prompt, d, f, args.experts, args.top_k, args.shared)) == 0:
        ap.error("--dims are multiples of 64, --top-k at most --experts, and these with --shared (from 0) at most 1024")
    gate = None
    if args.balance_steps < 0 or not 0 <= args.balance_rate < float("inf"):
        ap.error("--balance-steps and --balance-rate are not negative")
    if (args.scores, args.groups, args.groups_kept, args.group_best, args.scale) != ("softmax", 1, None, 1, 1.0) or args.balance_steps:
        gate = B.Gate(args.scores, args.groups, args.groups_kept, args.group_best, args.scale)
        if args.groups < 1 or args.experts % args.groups or not 1 <= gate.groups_kept <= args.groups:
            ap.error("--groups divide --experts, --groups-kept are at most as many")
        size = args.experts // args.groups
        if not 1 <= args.group_best <= min(2, size) or args.top_k > gate.groups_kept * size:
            ap.error("--group-best is 1 or 2 of a group's experts, --top-k at most those of --groups-kept")
        if not 0 < args.scale < float("inf"):
            ap.error("--scale is positive")
    if args.norm and d > B.NORM_COLS_MAX:
        ap.error(f"--dims: the norm takes up to {B.NORM_COLS_MAX}")
    if not torch.cuda.is_available():
        print("answering needs a GPU", file=sys.stderr)
        return 2
    print(json.dumps(run(d, f, args.experts, args.top_k, args.shared, args.prompt, args.batch, args.steps, gate=gate, norm=args.norm,
                         balance_steps=args.balance_steps, balance_rate=args.balance_rate)), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
