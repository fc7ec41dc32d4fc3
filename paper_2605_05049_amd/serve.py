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
from .layer import FewTokenBuffers, PromptMemory, layer_few_forward, layer_forward, layer_mxfp4_forward, on_stream, quantize_experts


class ServedLayer:
    """A layer that only answers: `layer(x)` for x [T, d_model] bf16, any T.  At most FEW_TOKENS_MAX tokens are answered by layer_few_forward,
    more by the grouped products.  `mxfp4`: the experts' weights are quantised here, and the bf16 ones are not kept; and a call with more than a few tokens
    quantises its rows and hidden activations to 4 bits on the way (its answers are 30 % off those of bf16, of random weights and rows, where a call
    with a few tokens, whose rows stay bf16, is 20 % off).  Without it everything is bf16.

    The buffers of a few tokens are made for their count at its first call and kept; what a call returns is theirs and is overwritten by the next
    call with as many tokens.  Longer calls share the memory of the longest so far, and each returns a tensor of its own.  Memory that a captured
    call uses stays as long as the layer.  Calls on one stream at a time; the memory is freed for others when all streams that had calls are past
    them."""

    def __init__(self, w_router, w_gate, w_up, w_down, top_k, n_shared=0, renorm=1, mxfp4=True, stream=None):
        E, d = w_router.shape
        n, f = E + n_shared, w_gate.shape[-1]
        for name, w, want in (("w_gate", w_gate, (n, d, f)), ("w_up", w_up, (n, d, f)), ("w_down", w_down, (n, f, d))):
            if tuple(w.shape) != want:
                raise ValueError(f"{name} {tuple(w.shape)}: expected {want}")
        self.w_router, self.mxfp4 = w_router, mxfp4
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
            buf = self._few[T] = FewTokenBuffers(s, self.w_router.device)
        return buf

    def __call__(self, x, stream=None):
        if x.dim() != 2 or x.shape[1] != self._fields[0]:
            raise ValueError(f"x {tuple(x.shape)}: expected [T, {self._fields[0]}]")
        import torch
        with on_stream(stream):
            buf = self.buffers(x.shape[0])
            if isinstance(buf, FewTokenBuffers):
                out = layer_few_forward(buf, x, self.weights, w_router=self.w_router)
                self._used(buf.streams, vars(buf).values())
                return out
            buf.out = torch.empty_like(buf.out)
            if self.mxfp4:
                out = layer_mxfp4_forward(buf, x, self.weights, w_router=self.w_router)
            else:
                out = layer_forward(buf, x, *self.weights, w_router=self.w_router)
            block = self._prompts.block
            self._used(self._prompts.streams, (block,))
            if torch.cuda.is_current_stream_capturing() and not any(b is block for b in self._captured):
                self._captured.append(block)
            return out

    def _used(self, streams, tensors):
        """What the call used, these tensors and the weights, is not to be handed out again before the current stream is past it.  (Once per stream: the
        allocator waits for what a stream has enqueued by the time the memory is freed.)"""
        import torch
        handle = B._stream(None)
        if handle in streams and handle in self._streams:
            return
        for seen, what in ((self._streams, (self.w_router, *self.weights)), (streams, tensors)):
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
    """The layer over the prompt, then `steps` steps of the prompt's last `batch` rows; (answers of the prompt, of every step)."""
    import torch
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


def run(d, f, experts, top_k, shared, prompt, batch, steps, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std: (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    n = experts + shared
    weights = [torch.stack([normal(*s, std=std) for _ in range(n)]) for s, std in (((d, f), d ** -0.5), ((d, f), d ** -0.5), ((f, d), f ** -0.5))]
    w_router, x = normal(experts, d, std=2 * d ** -0.5), normal(prompt, d, std=1.0)
    full = ServedLayer(w_router, *weights, top_k, shared, mxfp4=False)
    layer = ServedLayer(w_router, *weights, top_k, shared)
    ref, got = full(x).float(), layer(x).float()
    answer(layer, x, batch, steps)
    static = x[-batch:].clone()
    layer(static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step = layer(static)
    step_ref = full(static).float()
    graph.replay()
    step = step.float()
    off = lambda a, b: round(((a - b).norm() / b.norm()).item(), 4)  # noqa: E731
    return {"d_model": d, "d_ffn": f, "experts": experts, "shared": shared, "top_k": top_k, "prompt": prompt, "batch": batch,
            "weights_GB": round(sum(w.numel() * w.element_size() for w in layer.weights) / 1e9, 3),
            "bf16_weights_GB": round(sum(w.numel() * w.element_size() for w in weights) / 1e9, 3),
            "prompt_ms": round(_ms(lambda: layer(x), 5), 4), "bf16_prompt_ms": round(_ms(lambda: full(x), 5), 4),
            "step_us": round(1e3 * _ms(graph.replay, max(1, steps)), 2), "off_prompt": off(got, ref), "off_step": off(step, step_ref)}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--dims", default="2048x1408", help="d_model x d_ffn")
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--top-k", type=int, default=6)
    ap.add_argument("--shared", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=4096, help="tokens")
    ap.add_argument("--batch", type=int, default=1, help="tokens of a step")
    ap.add_argument("--steps", type=int, default=64)
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
    if not torch.cuda.is_available():
        print("answering needs a GPU", file=sys.stderr)
        return 2
    print(json.dumps(run(d, f, args.experts, args.top_k, args.shared, args.prompt, args.batch, args.steps)), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
