"""The operators together, as a MoE layer uses them: on the weights that a codec reconstructs, forwards and backwards."""
import pytest
import torch

from paper_2609_04609_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _layer(e, d, f, k, t, dtype="bf16", seed=1, **kw):
    from paper_2609_04609_b200 import runtime

    codec = runtime.LayerCodec.from_tensors([r * c for r, c in wl.olmoe_layer_shapes(e, d, f)], 4, dtype, 512, DEV)
    gen = wl.make_generator(seed, DEV)
    w = wl.init_weights(codec.weights_bytes // wl.VALUE_BYTES[dtype], dtype, gen, d**-0.5)
    codec.init_caches(w.view(torch.uint8))
    return codec.expert_layer(e, d, f, k, t, **kw), w.view(torch.uint8)


def _plain(layer, x, logits, bias, dout, score, renorm, scale):
    """The layer without any rounding, in 64 bits, gradients by autograd; the choice is the layer's own."""
    at = layer.experts[: x.shape[0]].long()
    x, logits = x.double().requires_grad_(), logits.double().requires_grad_()
    gate, up, down = (w.double().detach().clone().requires_grad_() for w in (layer.gate, layer.up, layer.down))
    s = logits.softmax(1) if score == "softmax" else logits.sigmoid()
    p = s.gather(1, at.clamp(min=0)) * (at >= 0)
    total = p.sum(1, keepdim=True)
    p = scale * (p / torch.where(total > 0, total, torch.ones_like(total)) if renorm else p)
    y = torch.zeros_like(x)
    for e in range(layer.n_experts):
        t, j = (at == e).nonzero(as_tuple=True)
        h = torch.nn.functional.silu(x[t] @ gate[e]) * (x[t] @ up[e])
        y = y.index_add(0, t, p[t, j, None] * (h @ down[e]))
    y.backward(dout.double())
    return y.detach(), x.grad, logits.grad, gate.grad, up.grad, down.grad


def _logits_size(layer, logits, dout, score, renorm, scale):
    from tests import moe_reference as ref

    n, k = logits.shape[0], layer.top_k
    o = layer.o[layer.row_of_slot[:n].long().clamp(min=0)].double().norm(dim=2) * (layer.row_of_slot[:n] >= 0)
    typical = (dout.double().norm(dim=1)[:, None] * o / layer.d_model**0.5).cpu()
    total = 0.0
    for j in range(k):
        dw = torch.zeros(n, k, dtype=torch.float64)
        dw[:, j] = typical[:, j]
        total += (ref.route_backward(logits.cpu(), layer.experts[:n], dw, score, renorm, scale) ** 2).sum()
    return float(total) ** 0.5


# A value rounded to e4m3 is off by at most 2^-4 of itself, 0.036 in the root of the mean square if its mantissa is anywhere.
# With errors that are independent of each other a product's sum is off by 0.036 * sqrt(2) = 0.05; silu(g) * u by up to 0.05 *
# sqrt(2) * 1.25 = 0.09; the output, with two more roundings, by 0.1.  The gradients have one or two products more: weights and
# inputs 0.14.  A weight's gradient is the product of a row of the output with its gradient, a sum of d terms of either sign: of
# the size |dout| |o| / sqrt(d), as its error is 0.1 times that, but not of that size for each token alone.  So the logits'
# gradient is measured by what gradients of just that size would make it, three times 0.1 for the one token of a batch of one.
OFF = {"y": 0.15, "dx": 0.2, "dlogits": 0.3, "dgate": 0.2, "dup": 0.2, "ddown": 0.2}


@pytest.mark.parametrize("e,d,f,k,t,dtype,score,renorm", [
    (8, 256, 128, 2, 100, "bf16", "softmax", False),
    (16, 384, 256, 4, 333, "bf16", "sigmoid", True),
    (4, 128, 128, 1, 1, "fp16", "softmax", False),
    (8, 256, 384, 3, 64, "fp32", "softmax", True),
])
def test_layer_forward_and_backward(e, d, f, k, t, dtype, score, renorm):
    from paper_2609_04609_b200 import ciera

    scale = 2.0 if renorm else 1.0
    layer, w = _layer(e, d, f, k, t + 7, dtype, score=ciera.SCORE_SIGMOID if score == "sigmoid" else ciera.SCORE_SOFTMAX,
                      renormalise=renorm, scale=scale)
    layer.step(w)
    assert torch.equal(layer.codec.weights_out, w)
    gen = wl.make_generator(2, DEV)
    for n in (t, max(1, t // 3)):  # a second, smaller batch in the same buffers
        x = torch.randn(n, d, generator=gen, device=DEV).to(layer.dtype)
        logits = torch.randn(n, e, generator=gen, device=DEV).to(layer.dtype)
        if n > 2:
            logits[1] = float("-inf")  # a token that goes nowhere
        bias = torch.rand(e, generator=gen, device=DEV) * 0.1 if score == "sigmoid" else None
        dout = torch.randn(n, d, generator=gen, device=DEV).to(layer.dtype)
        y = layer.forward(x, logits, bias)
        got = (y,) + layer.backward(dout)
        torch.cuda.synchronize()
        layer.check_status()
        plain_logits = logits.clone()
        if n > 2:
            plain_logits[1] = 0.0
            assert (y[1] == 0).all() and (got[1][1] == 0).all() and (got[2][1] == 0).all()
        want = _plain(layer, x, plain_logits, bias, dout, score, renorm, scale)
        for name, a, b in zip(OFF, got, want):
            size = float(b.norm())
            if name == "dlogits":
                size = _logits_size(layer, plain_logits, dout, score, renorm, scale)
            off = float((a.double() - b).norm()) / size if size else float(a.double().norm())
            assert off < OFF[name], (name, off)


def test_each_stage_is_the_operator_on_the_stage_before():
    """Every buffer between two operators holds what the definition gives for the buffers before it."""
    from tests import moe_reference as ref

    e, d, f, k, t = 8, 256, 128, 2, 150
    layer, w = _layer(e, d, f, k, t)
    layer.step(w)
    gen = wl.make_generator(3, DEV)
    x = torch.randn(t, d, generator=gen, device=DEV).bfloat16()
    logits = torch.randn(t, e, generator=gen, device=DEV)
    y = layer.forward(x, logits)
    torch.cuda.synchronize()
    ids, p = ref.route(logits.cpu(), None, k, "softmax")
    assert (layer.experts.cpu().numpy() == ids).all()
    starts, _, ros, _ = ref.layout(torch.from_numpy(ids), e)
    assert layer.starts.tolist() == starts and layer.row_of_slot.reshape(-1).tolist() == ros
    used = starts[-1]
    rows = torch.tensor(ros, device=DEV)
    for i in range(e):
        q, s = ref.quantize_blocks(layer.gate[i].double().cpu().numpy())
        assert (ref.e4m3_values()[layer.w1_t[i, :, :f].view(torch.uint8).cpu().numpy()] == q).all()
        assert (ref.e4m3_values()[layer.w1[i, :f].view(torch.uint8).cpu().numpy()] == q.T).all()
        assert (layer.w1_s[i, : f // 128].cpu().numpy() == s.T).all()
    xv = ref.operand_values(layer.x_q[:used], layer.x_s)
    want = torch.zeros(used, d, dtype=torch.float64, device=DEV)
    q, s = ref.quantize_rows(x.double().cpu().numpy())
    value = torch.from_numpy(q).to(DEV) * torch.exp2(torch.from_numpy(s).to(DEV).double() - 127).t().repeat_interleave(128, 1)
    want[rows] = value.repeat_interleave(k, 0)
    assert torch.equal(xv, want)
    w1 = ref.matrix_values(layer.w1, layer.w1_s)
    for i in range(e):
        lo, hi = starts[i], starts[i + 1]
        h = xv[lo:hi] @ w1[i].t()
        size = xv[lo:hi].abs() @ w1[i].abs().t()
        assert ((layer.h[lo:hi].double() - h).abs() <= (d + 2) * 2.0**-24 * size + 2.0**-8 * h.abs()).all()
    o = layer.o[rows].double().view(t, k, d)
    terms = torch.from_numpy(p).to(DEV)[:, :, None] * o
    assert ((y.double() - terms.sum(1)).abs() <= (e + 24) * 2.0**-24 * terms.abs().sum(1) + 2.0**-8 * terms.sum(1).abs()).all()


def test_layer_in_a_graph_follows_new_weights_and_tokens():
    """Gather, rounding, forward and backward in one captured graph, replayed on other weights and another routing."""
    e, d, f, k, t = 8, 256, 128, 2, 64
    layer, w = _layer(e, d, f, k, t)
    gen = wl.make_generator(5, DEV)
    x = torch.randn(t, d, generator=gen, device=DEV).bfloat16()
    logits = torch.randn(t, e, generator=gen, device=DEV)
    dout = torch.randn(t, d, generator=gen, device=DEV).bfloat16()
    w = w.clone()

    def run():
        layer.step(w)
        y = layer.forward(x, logits)
        return (y,) + layer.backward(dout)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for seed in (6, 7):
        g = wl.make_generator(seed, DEV)
        w.copy_(wl.init_weights(w.numel() // 2, "bf16", g, 0.05).view(torch.uint8))
        logits.copy_(torch.randn(t, e, generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        layer.codec.check_status()
        layer.check_status()
        got = [o.clone() for o in outs]
        again = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_layer_without_tokens():
    layer, w = _layer(4, 128, 128, 2, 8)
    layer.step(w)
    y = layer.forward(torch.zeros(0, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(0, 4, device=DEV))
    grads = layer.backward(torch.zeros_like(y))
    assert y.shape == (0, 128) and all((g == 0).all() for g in grads[2:])
