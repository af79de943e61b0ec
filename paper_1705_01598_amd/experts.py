"""A gated mixture-of-experts layer, forward and backward, on the library's operators (application layer).

Every token has ``slots`` experts; expert e maps a row x of ``width`` channels to

    w_out[e] @ (silu(g) * u),   (g, u) = the halves of w_in[e] @ x,

and the token's result is the weighted sum over its experts.  One forward pass is a sort of the assignments by
expert, the two products with the gated activation between them and the combination of the rows; the first product
reads tokens through the sorted order, so rows are never gathered into a buffer.  For the backward pass the layer
keeps the input and the gates in 8 bits (``tperm_checkpoint_store``, ``tperm_gated_forward``); the input's rows
are multiplied out of their codes.  A program that only asks for answers calls ``answer``, which keeps nothing and takes few tokens through
two kernels (or a third that joins their shares), with matrices as they are or held in 4 bits (``hold``); ``route`` chooses the experts and their weights from a
router's scores, ``route_backward`` takes the weights' gradient back to them.  Everything here is argument bookkeeping around the calls of
``include/tperm_experts.h`` and ``include/tperm_decode.h``; tensors are dense and contiguous, on the layer's GPU, and work is enqueued on
that GPU's current stream, whichever GPU is the current one (a layer is used on one stream at a time).
"""
from __future__ import annotations

import contextlib
import itertools
from typing import Dict, NamedTuple, Tuple

_HERE = contextlib.nullcontext()
_NAMES = {"torch.float32": "f32", "torch.float16": "f16", "torch.bfloat16": "bf16"}


class HeldMatrices(NamedTuple):
    """A layer's matrices in 4 bits, as tperm_four_bit_store writes them: for w_in and w_out codes [experts, rows, 16 * groups] and
    scales [experts, rows, groups], a group to every 32 elements of a row."""
    w_in: "torch.Tensor"        # noqa: F821
    in_scales: "torch.Tensor"   # noqa: F821
    w_out: "torch.Tensor"       # noqa: F821
    out_scales: "torch.Tensor"  # noqa: F821


class ExpertLayer:
    """The operators of one layer shape, and what a forward pass keeps for the backward pass: the maps, the input and the
    gates in 8 bits and the rows that the experts gave, in buffers that are reused for the largest number of tokens met so far, so that a
    forward pass overwrites what the one before it kept.  What a pass needs beside that goes back to the allocator
    at its end.  ``device`` without a number ("cuda")
    becomes that of the first tensors; from then on tensors of another device are refused."""

    def __init__(self, experts: int, slots: int, width: int, hidden: int, dtype, device="cuda"):
        import torch
        from . import binding as B
        self._torch, self._B = torch, B
        if str(dtype) not in _NAMES:
            raise ValueError("float32, float16 or bfloat16 only")
        if not (1 <= experts <= B.EXPERTS_MAX and 1 <= slots <= B.SLOTS_MAX and width >= 1 and hidden >= 1 and max(width, 2 * hidden) <= B.WIDTH_MAX):
            raise ValueError("sizes outside the limits of tperm_experts.h")
        self.experts, self.slots, self.width, self.hidden, self.dtype = experts, slots, width, hidden, dtype
        self._type = B.TYPES[_NAMES[str(dtype)]]
        self._device = torch.device(device)
        self._size = dtype.itemsize
        self._room, self._b, self._at = -1, {}, {}
        self._kept = None

    def _buffers(self, tokens: int) -> Dict[str, int]:
        if tokens > self._room:
            torch, B = self._torch, self._B
            rows, w, h = tokens * self.slots, self.width, self.hidden
            new = lambda *shape, dtype=self.dtype: torch.empty(*shape, dtype=dtype, device=self._device)  # noqa: E731
            i32, u8 = torch.int32, torch.uint8
            self._b = {"offsets": new(self.experts + 1, dtype=i32), "source": new(rows, dtype=i32), "place": new(rows, dtype=i32),
                       "x_codes": new(tokens * w, dtype=u8), "x_scales": new(tokens * B.checkpoint_blocks(w), dtype=u8),
                       "gate_codes": new(rows * 2 * h, dtype=u8), "gate_scales": new(rows * 2 * B.checkpoint_blocks(h), dtype=u8),
                       "rows": new(rows, w)}
            self._at = {k: t.data_ptr() for k, t in self._b.items()}
            self._room = tokens
        return self._at

    def _scratch(self, *sizes: int):
        """One buffer for a pass's own arrays of so many bytes each: the buffer, and where each of them starts in it."""
        room = [n + 255 & ~255 for n in sizes]
        buffer = self._torch.empty(sum(room), dtype=self._torch.uint8, device=self._device)
        return buffer, *itertools.accumulate(room[:-1], initial=buffer.data_ptr())

    def kept_bytes(self) -> int:
        """Bytes of GPU memory that the layer holds between its passes."""
        return sum(t.numel() * t.element_size() for t in self._b.values())

    def _check(self, name: str, t, shape: Tuple[int, ...], dtype, device) -> None:
        if tuple(t.shape) != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {shape} on {device} is wanted")

    def _gpu(self):
        """The layer's GPU as the current one, while calls are enqueued."""
        if self._device.type != "cuda":
            raise ValueError("the layer computes on a GPU: no host tensors")
        return _HERE if self._torch.cuda.current_device() == self._device.index else self._torch.cuda.device(self._device)

    def _device_of(self, t):
        return t.device if self._device.index is None and t.device.type == self._device.type else self._device

    def route(self, scores, over_all: bool = False):
        """The experts of every token and their weights from scores [tokens, experts] (float32, float16 or bfloat16): those with the
        largest scores, and the softmax over these, or with over_all their part of the softmax over all.  Scores of minus infinity
        or NaN bar an expert; a slot that finds none holds -1 and the weight 0."""
        torch, B = self._torch, self._B
        if str(scores.dtype) not in _NAMES:
            raise ValueError("scores: float32, float16 or bfloat16 only")
        tokens, device = scores.shape[0], self._device_of(scores)
        self._check("scores", scores, (tokens, self.experts), scores.dtype, device)
        self._device = device
        expert = torch.empty(tokens, self.slots, dtype=torch.int32, device=device)
        weights = torch.empty(tokens, self.slots, dtype=torch.float32, device=device)
        with self._gpu():
            B.tperm_expert_route(scores.data_ptr(), self.experts, expert.data_ptr(), weights.data_ptr(), tokens, self.slots, self.experts, over_all,
                                 B.TYPES[_NAMES[str(scores.dtype)]], torch.cuda.current_stream().cuda_stream)
        return expert, weights

    def route_backward(self, grad_weights, scores, expert, weights, over_all: bool = False):
        """The gradient of the scores from that of the weights (float32), which backward() returns; the other arguments as route() took
        and gave them."""
        torch, B = self._torch, self._B
        if str(scores.dtype) not in _NAMES:
            raise ValueError("scores: float32, float16 or bfloat16 only")
        tokens, device = scores.shape[0], self._device_of(scores)
        self._check("scores", scores, (tokens, self.experts), scores.dtype, device)
        self._check("expert", expert, (tokens, self.slots), torch.int32, device)
        self._check("weights", weights, (tokens, self.slots), torch.float32, device)
        self._check("grad_weights", grad_weights, (tokens, self.slots), torch.float32, device)
        self._device = device
        grad = torch.empty_like(scores)
        with self._gpu():
            B.tperm_expert_route_backward(grad_weights.data_ptr(), scores.data_ptr(), self.experts, expert.data_ptr(), weights.data_ptr(), grad.data_ptr(),
                                          self.experts, tokens, self.slots, self.experts, over_all, B.TYPES[_NAMES[str(scores.dtype)]],
                                          torch.cuda.current_stream().cuda_stream)
        return grad

    def hold(self, w_in, w_out) -> HeldMatrices:
        """The matrices in 4 bits, for answer(): 17 bytes for 32 elements."""
        torch, B = self._torch, self._B
        e, w, h = self.experts, self.width, self.hidden
        device = self._device_of(w_in)
        self._check("w_in", w_in, (e, 2 * h, w), self.dtype, device)
        self._check("w_out", w_out, (e, w, h), self.dtype, device)
        self._device = device
        held = []
        with self._gpu():
            for m in (w_in, w_out):
                rows, width = m.shape[1:]
                groups = B.four_bit_groups(width)
                codes = torch.empty(e, rows, 16 * groups, dtype=torch.uint8, device=device)
                scales = torch.empty(e, rows, groups, dtype=torch.uint8, device=device)
                B.tperm_four_bit_store(m.data_ptr(), width, codes.data_ptr(), scales.data_ptr(), e * rows, width, self._type, torch.cuda.current_stream().cuda_stream)
                held += [codes, scales]
        return HeldMatrices(*held)

    def answer(self, x, expert, weights, w_in, w_out=None):
        """The layer's result as forward() gives it, with nothing kept for a backward pass and what a forward pass kept left as it is.  w_in and
        w_out are matrices, or w_in alone is what hold() gave.  Up to FEW_TOKENS tokens take kernels that read the named experts'
        matrices once for every 32 tokens that name them; more take the passes of forward().  For these, matrices in 4 bits are brought back to the
        layer's type in every call, all experts' and in memory of that size (128 experts of 2048 -> 2 x 1024 -> 2048 in 16 bits: 1.6 GB written and read);
        a program without that memory answers in parts of FEW_TOKENS tokens."""
        torch, B = self._torch, self._B
        e, k, w, h, t = self.experts, self.slots, self.width, self.hidden, self._type
        held = w_in if isinstance(w_in, HeldMatrices) else None
        if (held is None) == (w_out is None):
            raise ValueError("w_in and w_out, or held matrices alone")
        tokens = x.shape[0]
        rows = tokens * k
        device = self._device_of(x)
        self._check("x", x, (tokens, w), self.dtype, device)
        self._check("expert", expert, (tokens, k), torch.int32, device)
        self._check("weights", weights, (tokens, k), torch.float32, device)
        if held is not None:
            for name, m, shape in zip(HeldMatrices._fields, held, ((e, 2 * h, 16 * B.four_bit_groups(w)), (e, 2 * h, B.four_bit_groups(w)),
                                                                   (e, w, 16 * B.four_bit_groups(h)), (e, w, B.four_bit_groups(h)))):
                self._check(name, m, shape, torch.uint8, device)
        else:
            self._check("w_in", w_in, (e, 2 * h, w), self.dtype, device)
            self._check("w_out", w_out, (e, w, h), self.dtype, device)
        self._device = device
        out = torch.empty_like(x)
        if tokens == 0:
            return out
        with self._gpu():
            s = torch.cuda.current_stream().cuda_stream
            if tokens <= B.FEW_TOKENS:
                matrices = (w_in.data_ptr(), None, w_out.data_ptr(), None) if held is None else tuple(m.data_ptr() for m in held)
                need = B.expert_few_workspace_bytes(tokens, k, e, w, h, t, held is not None)
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
                B.tperm_expert_few(x.data_ptr(), w, expert.data_ptr(), weights.data_ptr(), *matrices, out.data_ptr(), w, workspace.data_ptr(), need,
                                   tokens, k, e, w, h, t, s)
                return out
            size, need = self._size, B.expert_sort_workspace_bytes(rows, e)
            restored = (e * 2 * h * w * size, e * w * h * size) if held is not None else (0, 0)
            scratch, gates, hidden, back, sort, offsets, source, place, in_matrices, out_matrices = self._scratch(
                rows * 2 * h * size, rows * h * size, rows * w * size, need, 4 * (e + 1), 4 * rows, 4 * rows, *restored)
            if held is not None:
                B.tperm_four_bit_load(held.w_in.data_ptr(), held.in_scales.data_ptr(), in_matrices, w, e * 2 * h, w, t, s)
                B.tperm_four_bit_load(held.w_out.data_ptr(), held.out_scales.data_ptr(), out_matrices, h, e * w, h, t, s)
            else:
                in_matrices, out_matrices = w_in.data_ptr(), w_out.data_ptr()
            B.tperm_expert_sort(expert.data_ptr(), tokens, k, e, offsets, source, place, sort, need, s)
            B.tperm_expert_product(x.data_ptr(), w, tokens, source, k, offsets, in_matrices, True, gates, 2 * h, rows, e, w, 2 * h, t, s)
            B.tperm_gated_forward(gates, 2 * h, hidden, h, None, None, rows, h, t, s)
            B.tperm_expert_product(hidden, h, rows, None, 1, offsets, out_matrices, True, back, w, rows, e, h, w, t, s)
            B.tperm_expert_combine(back, w, place, offsets, weights.data_ptr(), out.data_ptr(), w, tokens, k, e, w, t, s)
        return out

    def forward(self, x, expert, weights, w_in, w_out):
        """The layer's result for x [tokens, width]; expert [tokens, slots] int32 (a number outside 0 .. experts-1 names
        none), weights [tokens, slots] float32, w_in [experts, 2 * hidden, width], w_out [experts, width, hidden]."""
        torch, B = self._torch, self._B
        e, k, w, h, t = self.experts, self.slots, self.width, self.hidden, self._type
        tokens = x.shape[0]
        rows = tokens * k
        device = self._device_of(x)
        self._check("x", x, (tokens, w), self.dtype, device)
        self._check("expert", expert, (tokens, k), torch.int32, device)
        self._check("weights", weights, (tokens, k), torch.float32, device)
        self._check("w_in", w_in, (e, 2 * h, w), self.dtype, device)
        self._check("w_out", w_out, (e, w, h), self.dtype, device)
        self._device = device
        out = torch.empty_like(x)
        if tokens == 0:
            self._kept = (tokens, weights, w_in, w_out)
            return out
        with self._gpu():
            self._kept = None       # the buffers of the pass before are overwritten from here on, whether this one succeeds or not
            b = self._buffers(tokens)
            need = B.expert_sort_workspace_bytes(rows, e)
            scratch, gates, hidden, sort = self._scratch(rows * 2 * h * self._size, rows * h * self._size, need)    # held to the last call
            s = torch.cuda.current_stream().cuda_stream
            B.tperm_expert_sort(expert.data_ptr(), tokens, k, e, b["offsets"], b["source"], b["place"], sort, need, s)
            B.tperm_checkpoint_store(x.data_ptr(), w, b["x_codes"], b["x_scales"], tokens, w, t, s)
            B.tperm_expert_product(x.data_ptr(), w, tokens, b["source"], k, b["offsets"], w_in.data_ptr(), True, gates, 2 * h, rows, e, w, 2 * h, t, s)
            B.tperm_gated_forward(gates, 2 * h, hidden, h, b["gate_codes"], b["gate_scales"], rows, h, t, s)
            B.tperm_expert_product(hidden, h, rows, None, 1, b["offsets"], w_out.data_ptr(), True, b["rows"], w, rows, e, h, w, t, s)
            B.tperm_expert_combine(b["rows"], w, b["place"], b["offsets"], weights.data_ptr(), out.data_ptr(), w, tokens, k, e, w, t, s)
        self._kept = (tokens, weights, w_in, w_out)
        return out

    def backward(self, grad, grad_w_in, grad_w_out, accumulate: bool = True):
        """Gradients of the last forward pass from grad, that of its result: returns those of x and weights, and puts
        (accumulate: adds) those of the matrices to grad_w_in and grad_w_out, float32 tensors of the matrices' shapes."""
        if self._kept is None:
            raise RuntimeError("backward() without a forward()")
        torch, B = self._torch, self._B
        e, k, w, h, t, f32 = self.experts, self.slots, self.width, self.hidden, self._type, self._B.TYPE_F32
        tokens, weights, w_in, w_out = self._kept
        rows = tokens * k
        self._check("grad", grad, (tokens, w), self.dtype, self._device)
        self._check("grad_w_in", grad_w_in, (e, 2 * h, w), torch.float32, self._device)
        self._check("grad_w_out", grad_w_out, (e, w, h), torch.float32, self._device)
        grad_x, grad_weights = torch.empty_like(grad), torch.empty_like(weights)
        self._kept = None           # what it reads is overwritten, and the matrices' gradients must not be added to twice
        if tokens == 0:
            if not accumulate:
                grad_w_in.zero_(), grad_w_out.zero_()
            return grad_x, grad_weights
        with self._gpu():
            b = self._buffers(tokens)
            # the hidden rows again, for their matrix, take the rows' place where they fit
            size, fits = self._size, h <= w
            scratch, grad_rows, hidden, gates, again = self._scratch(rows * w * size, rows * h * size, rows * 2 * h * size, 0 if fits else rows * h * size)
            again = b["rows"] if fits else again
            s = torch.cuda.current_stream().cuda_stream
            B.tperm_expert_combine_backward(grad.data_ptr(), w, b["rows"], w, b["place"], b["offsets"], weights.data_ptr(), grad_rows, w,
                                            grad_weights.data_ptr(), tokens, k, e, w, t, s)
            # to the hidden rows: the same matrices, the other index summed
            B.tperm_expert_product(grad_rows, w, rows, None, 1, b["offsets"], w_out.data_ptr(), False, hidden, h, rows, e, w, h, t, s)
            B.tperm_gated_backward(hidden, h, b["gate_codes"], b["gate_scales"], gates, 2 * h, again, h, rows, h, t, s)
            B.tperm_expert_weight_gradient(again, h, None, rows, None, 1, grad_rows, w, b["offsets"], grad_w_out.data_ptr(), f32, True, accumulate,
                                           rows, e, h, w, t, s)
            B.tperm_expert_weight_gradient(b["x_codes"], w, b["x_scales"], tokens, b["source"], k, gates, 2 * h, b["offsets"], grad_w_in.data_ptr(), f32, True,
                                           accumulate, rows, e, w, 2 * h, t, s)
            B.tperm_expert_product(gates, 2 * h, rows, None, 1, b["offsets"], w_in.data_ptr(), False, grad_rows, w, rows, e, 2 * h, w, t, s)
            B.tperm_expert_combine(grad_rows, w, b["place"], b["offsets"], None, grad_x.data_ptr(), w, tokens, k, e, w, t, s)
        return grad_x, grad_weights

    def kept_gates(self):
        """[g, u] of the sorted rows as the backward pass will see them, in float32 (the values that the codes stand for)."""
        if self._kept is None:
            raise RuntimeError("no forward pass is kept")
        torch, B = self._torch, self._B
        rows, h = self._kept[0] * self.slots, self.hidden
        blocks = B.checkpoint_blocks(h)
        # g and u of a row are checkpoints beside each other: as 2 * rows rows of h
        out = torch.empty(rows, 2 * h, dtype=torch.float32, device=self._device)
        if rows == 0:
            return out
        assert self._b["gate_scales"].numel() >= rows * 2 * blocks
        with self._gpu():
            b = self._buffers(self._kept[0])
            B.tperm_checkpoint_load(b["gate_codes"], b["gate_scales"], out.data_ptr(), h, 2 * rows, h, B.TYPE_F32, torch.cuda.current_stream().cuda_stream)
        return out


def _bench(argv=None):
    """Times a layer's forward and backward pass, or with --answer its answers (synthetic tokens, random routing)."""
    import argparse
    import json

    import torch
    ap = argparse.ArgumentParser(description=_bench.__doc__)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--experts", type=int, default=32)
    ap.add_argument("--slots", type=int, default=4)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--dtype", choices=["f32", "f16", "bf16"], default="bf16")
    ap.add_argument("--reps", type=int, default=10)
    ap.add_argument("--answer", action="store_true", help="router and answer, nothing kept")
    ap.add_argument("--bits", type=int, choices=[4, 16, 32], help="with --answer: 4 holds the matrices in 4 bits")
    a = ap.parse_args(argv)
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[a.dtype]
    if a.bits not in (None, 4, 8 * dtype.itemsize) or (a.bits == 4 and not a.answer):
        ap.error("--bits: 4 with --answer, or those of the type")
    g = torch.Generator(device="cuda").manual_seed(1705)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    layer = ExpertLayer(a.experts, a.slots, a.width, a.hidden, dtype)
    x, grad = randn(a.tokens, a.width).to(dtype), randn(a.tokens, a.width).to(dtype)
    w_in = (randn(a.experts, 2 * a.hidden, a.width) / a.width ** 0.5).to(dtype)
    w_out = (randn(a.experts, a.width, a.hidden) / a.hidden ** 0.5).to(dtype)
    grad_w_in, grad_w_out = torch.zeros(w_in.shape, device="cuda"), torch.zeros(w_out.shape, device="cuda")
    scores = randn(a.tokens, a.experts)
    expert, weights = layer.route(scores)

    def timed(f):
        f()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(a.reps):
            f()
        end.record()
        torch.cuda.synchronize()
        return begin.elapsed_time(end) / a.reps

    def both():
        layer.forward(x, expert, weights, w_in, w_out)
        layer.backward(grad, grad_w_in, grad_w_out)

    if a.answer:
        matrices = layer.hold(w_in, w_out) if a.bits == 4 else (w_in, w_out)
        named = int(expert.unique().numel())
        size = 3 * a.hidden * a.width * (17 / 32 if a.bits == 4 else dtype.itemsize)
        each = timed(lambda: layer.answer(x, *layer.route(scores), *([matrices] if a.bits == 4 else matrices)))
        print(json.dumps({"metric": "mixture-of-experts layer, router and answer", "tokens": a.tokens, "experts": a.experts, "slots": a.slots, "width": a.width,
                          "hidden": a.hidden, "dtype": a.dtype, "bits": a.bits or 8 * dtype.itemsize, "answer_ms": round(each, 4), "experts_named": named,
                          "matrices_tb_per_s": round(named * size / each / 1e9, 3)}), flush=True)
        return
    forward = timed(lambda: layer.forward(x, expert, weights, w_in, w_out))
    total = timed(both)
    flops = 2 * a.tokens * a.slots * 3 * a.hidden * a.width
    print(json.dumps({"metric": "mixture-of-experts layer, forward and backward", "tokens": a.tokens, "experts": a.experts, "slots": a.slots, "width": a.width,
                      "hidden": a.hidden, "dtype": a.dtype, "forward_ms": round(forward, 4), "forward_backward_ms": round(total, 4),
                      "forward_tflops": round(flops / forward / 1e9, 1), "forward_backward_tflops": round(3 * flops / total / 1e9, 1),
                      "kept_bytes_per_token": round(layer.kept_bytes() / a.tokens)}), flush=True)


if __name__ == "__main__":
    _bench()
