"""The computation of a MoE layer on the expert weights that a ``LayerCodec`` reconstructs.

Plumbing only, as in ``runtime``: torch allocates the buffers, every operation is a call into the library.  The products run
in 8-bit floating point with a power of two for each block of 128 values, forwards and backwards; what is summed or handed
from one product to the next is kept in the weights' type, gradients of weights in fp32.  A layer that only answers may have them
in 4 bits with a power of two for each 32 values, and has one call for a few tokens, whichever its weights are in.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional

import torch

from . import ciera
from .workloads import TORCH_DTYPES, VALUE_BYTES

BLOCK = ciera.FP8_BLOCK


def _operand(device, *shape):
    return torch.zeros(*shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)


def _bytes(device, *shape):
    return torch.zeros(*shape, dtype=torch.uint8, device=device)


def _atoms(device, *shape):
    """Scale bytes of a 4-bit operand [..., rows, cols]."""
    rows, cols = shape[-2:]
    return torch.full((*shape[:-2], -(-rows // BLOCK), -(-cols // BLOCK), ciera.FP4_ATOM), 127, dtype=torch.uint8, device=device)


class ExpertLayer:
    """``n_experts`` experts, each ``down(silu(gate(x)) * up(x))``, of which every token uses ``top_k``.

    ``codec`` holds the experts' matrices in the order gate, up (``d_model`` x ``d_ff``), down (``d_ff`` x ``d_model``), expert by
    expert (``workloads.olmoe_layer_shapes``), each in one piece.  ``refresh`` rounds what the codec has reconstructed
    (``step`` does a gather and that); ``forward`` and ``backward`` then work on up to ``max_tokens`` tokens.  The buffers
    belong to the layer, so one forward pass at a time can be waiting for its backward pass, and passes on different streams are put
    in order by the caller.  With ``stream`` a pass runs there whole: its results are allocated there too, and its inputs are kept
    from reuse until it is done with them.

    ``weight_bits=4`` (with ``training=False``): weights and rows in 4 bits, half the bytes and twice the rate, one bit behind the
    point.  ``forward_tokens`` is the pass of a few tokens (``ciera.EXPERT_TOKENS_MAX``) in one call that reads each reached
    expert's weights once; rows are not rounded to 8 or 4 bits there, so it is the more exact of the two.
    """

    def __init__(self, codec, n_experts: int, d_model: int, d_ff: int, top_k: int, max_tokens: int,
                 score: int = ciera.SCORE_SOFTMAX, n_groups: int = 1, top_groups: int = 1, group_best: int = 2,
                 renormalise: bool = False, scale: float = 1.0, training: bool = True, weight_bits: int = 8):
        if weight_bits not in (8, 4) or (weight_bits == 4 and training):
            raise ValueError("weight_bits is 8, or 4 with training=False: gradients take 8 bits")
        if d_model % BLOCK or d_ff % BLOCK or d_model < 1 or d_ff < 1:
            raise ValueError(f"d_model and d_ff are multiples of {BLOCK}")
        if max_tokens < 1 or n_experts < 1:
            raise ValueError("at least one token and one expert")
        if codec.weights_out is None:
            raise ValueError("the codec has no buffer for reconstructed weights")
        self.codec, self.device = codec, codec.device
        self.n_experts, self.d_model, self.d_ff, self.top_k, self.max_tokens = n_experts, d_model, d_ff, top_k, max_tokens
        self.training, self.weight_bits = training, weight_bits
        self.dtype = TORCH_DTYPES[codec.dtype_name]
        self.config = ciera.RouteConfig(n_experts=n_experts, top_k=top_k, n_groups=n_groups, top_groups=top_groups,
                                        group_best=group_best, score=score, renormalise=int(renormalise), scale=scale)
        # the matrices as they lie in the codec's buffer
        size, value = d_model * d_ff, VALUE_BYTES[codec.dtype_name]
        off = codec.units["weights_off"].astype("int64")
        n = codec.units["n_values"].astype("int64") * value
        if int(n.sum()) != 3 * n_experts * size * value or (off[1:] != off[:-1] + n[:-1]).any() or off[0] != 0:
            raise ValueError("the codec's table is not gate, up and down of every expert, each in one piece and in order")
        flat = codec.weights_out[: 3 * n_experts * size * value].view(self.dtype)
        self.gate = flat.as_strided((n_experts, d_model, d_ff), (3 * size, d_ff, 1), flat.storage_offset())
        self.up = flat.as_strided((n_experts, d_model, d_ff), (3 * size, d_ff, 1), flat.storage_offset() + size)
        self.down = flat.as_strided((n_experts, d_ff, d_model), (3 * size, d_model, 1), flat.storage_offset() + 2 * size)
        dev, e, d, f, b = self.device, n_experts, d_model, d_ff, BLOCK
        # gate and up side by side, down: rows of outputs (forward) and rows of inputs (backward)
        four = weight_bits == 4
        if four:
            self.w1, self.w1_s = _bytes(dev, e, 2 * f, d // 2), _atoms(dev, e, 2 * f, d)
            self.w2, self.w2_s = _bytes(dev, e, d, f // 2), _atoms(dev, e, d, f)
        else:
            self.w1, self.w1_s = _operand(dev, e, 2 * f, d), _bytes(dev, e, 2 * f // b, d // b)
            self.w2, self.w2_s = _operand(dev, e, d, f), _bytes(dev, e, d // b, f // b)
            self.w1_t, self.w1_ts = _operand(dev, e, d, 2 * f), _bytes(dev, e, d // b, 2 * f // b)
            self.w2_t, self.w2_ts = _operand(dev, e, f, d), _bytes(dev, e, f // b, d // b)
        # per batch
        slots = max_tokens * top_k
        cap = ciera.expert_rows_capacity(slots, e)
        i32 = dict(dtype=torch.int32, device=dev)
        self.experts, self.row_of_slot = torch.zeros(max_tokens, top_k, **i32), torch.zeros(max_tokens, top_k, **i32)
        self.weights = torch.zeros(max_tokens, top_k, device=dev)
        self.starts, self.counts, self.slot_of_row = torch.zeros(e + 1, **i32), torch.zeros(e, **i32), torch.zeros(cap, **i32)
        self.workspace = _bytes(dev, max(ciera.expert_layout_workspace_bytes(slots, e), 16))
        self.status = torch.zeros(1, **i32)
        if four:
            self.x_q, self.x_s = _bytes(dev, cap, d // 2), _atoms(dev, cap, d)
            self.a_q, self.a_s = _bytes(dev, cap, f // 2), _atoms(dev, cap, f)
        else:
            self.x_q, self.x_s = _operand(dev, cap, d), _bytes(dev, d // b, cap)
            self.a_q, self.a_s = _operand(dev, cap, f), _bytes(dev, f // b, cap)
        self.h = torch.zeros(cap, 2 * f, dtype=self.dtype, device=dev)
        self.few = min(max_tokens, ciera.EXPERT_TOKENS_MAX)  # tokens of forward_tokens
        self.few_workspace = _bytes(dev, ciera.expert_tokens_workspace_bytes(self.config, self.few, d, f))
        self.o = torch.zeros(cap, d, dtype=self.dtype, device=dev)
        if training:
            rb = cap // b
            self.x_t, self.x_ts = _operand(dev, d, cap), _bytes(dev, rb, d)
            self.a_t, self.a_ts = _operand(dev, f, cap), _bytes(dev, rb, f)
            self.do_q, self.do_s = _operand(dev, cap, d), _bytes(dev, d // b, cap)
            self.do_t, self.do_ts = _operand(dev, d, cap), _bytes(dev, rb, d)
            self.da = torch.zeros(cap, f, dtype=self.dtype, device=dev)
            self.dh_q, self.dh_s = _operand(dev, cap, 2 * f), _bytes(dev, 2 * f // b, cap)
            self.dh_t, self.dh_ts = _operand(dev, 2 * f, cap), _bytes(dev, rb, 2 * f)
            self.dx_rows = torch.zeros(cap, d, dtype=self.dtype, device=dev)
            self.dweights = torch.zeros(max_tokens, top_k, device=dev)
        self._batch = None
        if not torch.cuda.is_current_stream_capturing():  # the buffers are zeros before any stream writes them
            torch.cuda.current_stream(dev).synchronize()

    # -- weights ----------------------------------------------------------------------------------
    def refresh(self, stream=None) -> None:
        """Rounds the codec's reconstructed weights, both orientations (in 4 bits the one that forward passes need)."""
        if self.weight_bits == 4:
            f, lines = self.d_ff, self.d_ff // BLOCK
            ciera.fp4_quantize_matrices(self.gate, qt=self.w1[:, :f], scales_t=self.w1_s[:, :lines], stream=stream)
            ciera.fp4_quantize_matrices(self.up, qt=self.w1[:, f:], scales_t=self.w1_s[:, lines:], stream=stream)
            ciera.fp4_quantize_matrices(self.down, qt=self.w2, scales_t=self.w2_s, stream=stream)
            return
        f, fb = self.d_ff, self.d_ff // BLOCK
        for x, lo, lob in ((self.gate, 0, 0), (self.up, f, fb)):
            ciera.fp8_quantize_blocks(x, self.w1_t[:, :, lo : lo + f], self.w1_ts[:, :, lob : lob + fb], self.w1[:, lo : lo + f],
                                      self.w1_s[:, lob : lob + fb], stream)
        ciera.fp8_quantize_blocks(self.down, self.w2_t, self.w2_ts, self.w2, self.w2_s, stream)

    def step(self, weights: torch.Tensor, stream=None) -> None:
        """Gathers new weights (``LayerCodec.step``) and rounds them."""
        self.codec.step(weights, stream=stream)
        self.refresh(stream)

    # -- one batch --------------------------------------------------------------------------------
    def _rows(self, t: int) -> int:
        return ciera.expert_rows_capacity(t * self.top_k, self.n_experts)

    def _on(self, stream, *inputs):
        """The stream that a pass runs on and allocates from."""
        if stream is None:
            return nullcontext()
        for t in inputs:
            if t is not None:
                t.record_stream(stream)
        return torch.cuda.stream(stream)

    def forward(self, x: torch.Tensor, logits: torch.Tensor, bias: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """``x`` [T, d_model] in the weights' type, ``logits`` [T, n_experts]: the layer's output [T, d_model]."""
        t = x.shape[0]
        if t > self.max_tokens or tuple(x.shape) != (t, self.d_model) or x.dtype != self.dtype or logits.shape[0] != t:
            raise ValueError("x is [tokens, d_model] in the weights' type, with at most max_tokens tokens")
        self._batch = None  # (until this pass is on its way)
        with self._on(stream, x, logits, bias, out):
            out = torch.empty_like(x) if out is None else out
            if t:
                self._forward(x, logits, bias, out)
        self._batch = (x, logits)
        return out

    def _forward(self, x, logits, bias, out) -> None:
        t = x.shape[0]
        cap, k = self._rows(t), self.top_k
        experts, weights, rows = self.experts[:t], self.weights[:t], self.row_of_slot[:t]
        slots = self.slot_of_row[:cap]
        ciera.route(self.config, logits, bias, experts, weights)
        ciera.expert_layout(experts, self.n_experts, self.starts, self.counts, rows, slots, self.workspace)
        if self.weight_bits == 4:
            lines = cap // BLOCK
            ciera.fp4_quantize_rows(x, self.x_q[:cap], self.x_s[:lines], slot_of_row=slots, top_k=k, starts=self.starts)
            ciera.fp4_matmul(self.x_q[:cap], self.x_s[:lines], self.w1, self.w1_s, self.h[:cap], self.starts, status=self.status)
            ciera.fp4_quantize_rows(self.h[:cap], self.a_q[:cap], self.a_s[:lines], kind=ciera.SOURCE_SWIGLU, slot_of_row=slots,
                                    top_k=k, starts=self.starts)
            ciera.fp4_matmul(self.a_q[:cap], self.a_s[:lines], self.w2, self.w2_s, self.o[:cap], self.starts, status=self.status)
            ciera.expert_combine(self.o[:cap], rows, weights, out)
            return
        turned = self.training
        ciera.fp8_quantize_rows(x, self.x_q[:cap], self.x_s, self.x_t[:, :cap] if turned else None,
                                self.x_ts[: cap // BLOCK] if turned else None, slot_of_row=slots, top_k=k, starts=self.starts)
        ciera.fp8_matmul(self.x_q[:cap], self.x_s, self.w1, self.w1_s, self.h[:cap], self.starts, status=self.status)
        ciera.fp8_quantize_rows(self.h[:cap], self.a_q[:cap], self.a_s, self.a_t[:, :cap] if turned else None,
                                self.a_ts[: cap // BLOCK] if turned else None, kind=ciera.SOURCE_SWIGLU, slot_of_row=slots, top_k=k,
                                starts=self.starts)
        ciera.fp8_matmul(self.a_q[:cap], self.a_s, self.w2, self.w2_s, self.o[:cap], self.starts, status=self.status)
        ciera.expert_combine(self.o[:cap], rows, weights, out)

    def forward_tokens(self, x: torch.Tensor, logits: torch.Tensor, bias: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """``forward`` of at most ``few`` tokens by one call that reads each reached expert's weights once; nothing to go back
        through remains of it, nor of a ``forward`` before it.  The choice is in ``experts`` and ``weights`` as after ``forward``."""
        t = x.shape[0]
        if t > self.few or tuple(x.shape) != (t, self.d_model) or x.dtype != self.dtype or logits.shape[0] != t:
            raise ValueError("x is [tokens, d_model] in the weights' type, with at most `few` tokens")
        self._batch = None
        with self._on(stream, x, logits, bias, out):
            out = torch.empty_like(x) if out is None else out
            if t:
                ciera.expert_tokens(self.config, x, logits, bias, self.w1, self.w1_s, self.w2, self.w2_s, out, self.experts[:t],
                                    self.weights[:t], self.few_workspace, self.status)
        return out

    def backward(self, dout: torch.Tensor, stream=None):
        """Gradients of the last ``forward``: ``(dx, dlogits, dgate, dup, ddown)``, the last three in fp32 and the shapes of
        ``gate``, ``up`` and ``down``."""
        if not self.training or self._batch is None:
            raise RuntimeError("backward() follows a forward() of a layer made for training")
        x, logits = self._batch
        if dout.shape != x.shape or dout.dtype != self.dtype:
            raise ValueError("dout has the shape and type of x")
        with self._on(stream, x, logits, dout):
            return self._backward(x, logits, dout)

    def _backward(self, x, logits, dout):
        t, f, k = x.shape[0], self.d_ff, self.top_k
        new = lambda *shape: torch.empty(*shape, device=self.device)  # noqa: E731
        dx, dlogits = torch.empty_like(x), torch.empty_like(logits)
        dgate, dup = new(self.n_experts, self.d_model, f), new(self.n_experts, self.d_model, f)
        ddown = new(self.n_experts, f, self.d_model)
        if t == 0:
            return dx, dlogits, dgate.zero_(), dup.zero_(), ddown.zero_()
        cap, rows, slots = self._rows(t), self.row_of_slot[:t], self.slot_of_row[: self._rows(t)]
        rb = cap // BLOCK
        dweights = self.dweights[:t]
        ciera.expert_combine_backward(dout, self.o[:cap], rows, self.weights[:t], dweights)
        ciera.route_backward(self.config, logits, self.experts[:t], dweights, dlogits)
        ciera.fp8_quantize_rows(dout, self.do_q[:cap], self.do_s, self.do_t[:, :cap], self.do_ts[:rb], slot_of_row=slots, top_k=k,
                                row_weights=self.weights[:t], starts=self.starts)
        ciera.fp8_matmul(self.do_q[:cap], self.do_s, self.w2_t, self.w2_ts, self.da[:cap], self.starts, status=self.status)
        ciera.fp8_quantize_rows(self.h[:cap], self.dh_q[:cap], self.dh_s, self.dh_t[:, :cap], self.dh_ts[:rb],
                                kind=ciera.SOURCE_SWIGLU_BACKWARD, grad=self.da[:cap], slot_of_row=slots, top_k=k,
                                starts=self.starts)
        ciera.fp8_matmul(self.dh_q[:cap], self.dh_s, self.w1_t, self.w1_ts, self.dx_rows[:cap], self.starts, status=self.status)
        ciera.expert_combine(self.dx_rows[:cap], rows, None, dx)
        for a, a_s, b, b_s, out in ((self.x_t, self.x_ts, self.dh_t[:f], self.dh_ts[:, :f], dgate),
                                    (self.x_t, self.x_ts, self.dh_t[f:], self.dh_ts[:, f:], dup),
                                    (self.a_t, self.a_ts, self.do_t, self.do_ts, ddown)):
            ciera.fp8_matmul(a[:, :cap], a_s[:rb], b[:, :cap], b_s[:rb], out, self.starts, contract=True, status=self.status)
        return dx, dlogits, dgate, dup, ddown

    def check_status(self) -> None:
        """Waits for all streams' work and raises if a kernel of the layer reported an error since the last call."""
        torch.cuda.synchronize(self.device)
        s = int(self.status.item())
        if s != 0:
            self.status.zero_()
            self.few_workspace.zero_()  # (calls behind one that gave up give up too until then)
            torch.cuda.synchronize(self.device)
            raise ciera.CieraError("device status", s)
