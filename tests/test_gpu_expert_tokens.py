"""A whole MoE layer for a few tokens against 64 bits, alone and on the weights that a codec reconstructs."""
import numpy as np
import pytest
import torch

from tests import fp4_reference as f4
from tests import moe_reference as ref
from tests.test_gpu_fp8 import DTYPES, E4M3

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _stack(e, rows, cols, bits, seed):
    """Operand, scales and values (float64 on the device) of a stack of matrices."""
    from paper_2609_04609_b200 import ciera

    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randn(e, rows, cols, generator=g, device=DEV) * cols**-0.5
    w *= torch.exp2(torch.randint(-3, 4, (e, rows, 1), generator=g, device=DEV).float())  # scales differ
    if bits == 8:
        q = torch.zeros(e, rows, cols, dtype=torch.uint8, device=DEV).view(E4M3)
        s = torch.zeros(e, rows // 128, cols // 128, dtype=torch.uint8, device=DEV)
        ciera.fp8_quantize_blocks(w, q, s)
        return q, s, ref.matrix_values(q, s)
    q = torch.zeros(e, rows, cols // 2, dtype=torch.uint8, device=DEV)
    s = torch.zeros(e, rows // 128, cols // 128, 512, dtype=torch.uint8, device=DEV)
    ciera.fp4_quantize_matrices(w, q, s)
    v = torch.zeros(e, rows, cols, device=DEV)
    ciera.fp4_values(q, s, v)
    return q, s, v.double()


class Case:
    def __init__(self, t, e, k, d, f, bits, dtype="bf16", seed=1, score="softmax", logits_dtype=None, bias=False, **kw):
        from paper_2609_04609_b200 import ciera

        g = torch.Generator(device=DEV).manual_seed(seed)
        self.t, self.e, self.k, self.d, self.f, self.dt, self.bits = t, e, k, d, f, DTYPES[dtype], bits
        self.kw = {"top_k": k, **kw}
        self.score = score
        self.config = ciera.RouteConfig(n_experts=e, top_k=k, n_groups=kw.get("n_groups", 1), top_groups=kw.get("top_groups", 1),
                                        group_best=kw.get("group_best", 2), score=int(score == "sigmoid"),
                                        renormalise=int(kw.get("renormalise", False)), scale=kw.get("scale", 1.0))
        self.x = torch.randn(t, d, generator=g, device=DEV).to(self.dt)
        self.logits = torch.randn(t, e, generator=g, device=DEV).to(DTYPES[logits_dtype or dtype])
        self.bias = torch.rand(e, generator=g, device=DEV) * 0.1 if bias else None
        self.w1, self.w1_s, self.v1 = _stack(e, 2 * f, d, bits, seed + 1)
        self.w2, self.w2_s, self.v2 = _stack(e, d, f, bits, seed + 2)
        self.new()

    def new(self):
        from paper_2609_04609_b200 import ciera

        t, k = self.x.shape[0], self.k
        self.out = torch.full((t, self.d), 7.0, dtype=self.dt, device=DEV)
        self.experts = torch.full((t, k), 77, dtype=torch.int32, device=DEV)
        self.weights = torch.full((t, k), 7.0, device=DEV)
        n = ciera.expert_tokens_workspace_bytes(self.config, t, self.d, self.f)
        self.workspace = torch.zeros(n, dtype=torch.uint8, device=DEV)
        self.workspace[ciera.EXPERT_TOKENS_HEAD :] = 255  # (only the head has to be zero)
        return self

    def run(self, stream=None):
        from paper_2609_04609_b200 import ciera

        ciera.expert_tokens(self.config, self.x, self.logits, self.bias, self.w1, self.w1_s, self.w2, self.w2_s, self.out, self.experts,
                            self.weights, self.workspace, stream=stream)
        return self.out

    def check(self, tokens=None):
        from paper_2609_04609_b200 import ciera

        assert not self.workspace[: ciera.EXPERT_TOKENS_HEAD].any()
        self._check(tokens)

    def _check(self, tokens):
        """x and silu(g) * u go into the products in parts.  A part of 8 bits leaves 2^-4 of a value at most, one of 4 bits 1/3 of the
        largest of 32 and each further one a quarter of that; both are counted on the largest of 32.  Sums of d and f terms in 32
        bits, of which the tensor cores may cut off what is added, so two steps a term and 16 more for silu and the scales; the
        weights of the choice by 2^-20; one rounding at the end."""
        out, ids, weights, size = f4.layer(self.x.double(), self.logits, self.bias, self.v1, self.v2, self.kw, self.score)
        assert np.array_equal(self.experts.cpu().numpy(), ids)
        step = torch.finfo(self.dt).eps / 2
        parts = {8: {torch.float32: 5}, 4: {torch.float32: 10, torch.float16: 7}}[self.bits].get(self.dt, 3 if self.bits == 8 else 6)
        part = 2.0 ** (-4 * parts) if self.bits == 8 else 4.0 ** (1 - parts) / 3
        middle, left = self._sizes(ids, weights)
        tol = part * left + 2 * (self.d + self.f + self.k + 16) * 2.0**-24 * (size + middle) + 2.0**-20 * middle + step * out.abs()
        tol += 2.0**-24 if self.dt == torch.float16 else 1e-38
        off = (self.out.double() - out).abs()
        if tokens is not None:
            off, tol = off[tokens], tol[tokens]
        assert (off <= tol).all(), float((off / tol).max())

    def _sizes(self, ids, weights):
        """The sum of the magnitudes of the second product's terms, and what all values being off by the largest of their 32 would
        make of the output."""
        def largest(v):
            return v.abs().reshape(v.shape[0], -1, 32).amax(2).repeat_interleave(32, 1)

        s, left = (torch.zeros(self.x.shape, dtype=torch.float64, device=DEV) for _ in range(2))
        x = self.x.double()
        for e in range(self.e):
            t = np.nonzero(ids == e)[0]
            if not len(t):
                continue
            c = torch.from_numpy(np.abs(weights[ids == e])).to(DEV)[:, None]
            t = torch.from_numpy(t).to(DEV)
            h, hl = x[t] @ self.v1[e].T, largest(x[t]) @ self.v1[e].abs().T
            g, u = h[:, : self.f], h[:, self.f :]
            a = g / (1 + torch.exp(-g)) * u
            off = 1.1 * hl[:, : self.f] * u.abs() + g.abs() * hl[:, self.f :]
            s.index_add_(0, t, c * (a.abs() @ self.v2[e].abs().T))
            left.index_add_(0, t, c * ((off + largest(a)) @ self.v2[e].abs().T))
        return s, left


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,e,k,d,f,dtype", [
    (1, 8, 2, 128, 128, "bf16"), (1, 64, 8, 256, 128, "fp32"), (3, 4, 2, 384, 256, "fp16"), (8, 16, 4, 640, 384, "bf16"),
    (9, 4, 4, 1152, 128, "bf16"), (17, 2, 2, 256, 640, "fp32"), (64, 4, 2, 384, 256, "bf16"), (33, 64, 8, 128, 384, "fp16"),
    (64, 1, 1, 256, 128, "bf16"), (5, 6, 3, 2176, 128, "bf16"), (2, 3, 1, 4224, 256, "fp32"), (40, 3, 2, 2304, 2176, "bf16"),
    (64, 40, 32, 128, 128, "bf16"), (64, 1024, 32, 128, 128, "bf16"), (23, 2, 2, 256, 128, "fp32"), (12, 1, 1, 128, 256, "fp32"), (1, 300, 32, 128, 128, "fp16"),
    (3, 2, 2, 8192, 128, "bf16"),
])
def test_against_64_bits(t, e, k, d, f, dtype, bits):
    c = Case(t, e, k, d, f, bits, dtype)
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kw", [
    dict(score="sigmoid", n_groups=4, top_groups=2, bias=True, renormalise=True, scale=2.5), dict(score="sigmoid", logits_dtype="fp32"),
    dict(renormalise=True, logits_dtype="bf16", dtype="fp32"), dict(n_groups=8, top_groups=3, group_best=1),
])
def test_ways_of_routing(kw, bits):
    c = Case(11, 32, 4, 256, 128, bits, **{"dtype": "bf16", **kw})
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_tokens_with_fewer_experts_or_none(bits):
    c = Case(10, 6, 4, 256, 128, bits)
    c.logits[0] = float("-inf")
    c.logits[3, 1:] = float("-inf")
    c.logits[4, :3] = float("nan")
    c.run()
    c.check()
    assert (c.out[0] == 0).all() and (c.experts[0] == -1).all() and (c.experts[3, 1:] == -1).all()
    c.logits.fill_(float("-inf"))
    c.new().run()
    assert (c.out == 0).all() and (c.weights == 0).all()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_that_are_not_finite_stay_with_their_token(bits, dtype):
    c = Case(9, 4, 2, 256, 128, bits, dtype)
    c.run()
    clean = c.out.clone()
    c.x[2, 17], c.x[5, 200], c.x[6] = float("nan"), float("inf"), float("-inf")
    c.new().run()
    rest = [0, 1, 3, 4, 7, 8]
    assert torch.equal(c.out[rest], clean[rest])
    assert torch.isnan(c.out[2]).all() and not torch.isfinite(c.out[5]).any() and not torch.isfinite(c.out[6]).any()
    # an expert whose weights are not finite reaches the tokens that choose it
    c = Case(9, 4, 2, 256, 128, bits, dtype)
    if bits == 8:
        c.w1.view(torch.uint8)[1, 5] = 127
        c.w1_s[1] = 255
    else:
        c.w1_s[1, 0, 0, 16 * 5] = 255
    c.run()
    hit = (c.experts == 1).any(1)
    assert hit.any() and not hit.all()
    assert torch.isnan(c.out[hit]).all() and torch.equal(c.out[~hit], clean[~hit])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("power", [-60, -30, 30, 40])
def test_magnitudes(power, bits):
    """x so large or small that fp16 alone would not hold it, with a row of its own scale beside it."""
    c = Case(4, 4, 2, 384, 128, bits)
    c.x[1:] *= 2.0**power
    c.x[2, :64] *= 2.0**-20
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_strides_and_alignment(bits):
    """Rows that start at any value, matrices within larger ones, an output between other columns."""
    t, d, f = 7, 256, 128
    c = Case(t, 4, 2, d, f, bits)
    want = c.run().clone()
    big = torch.full((t, d + 5), 7.0, dtype=c.dt, device=DEV)
    big[:, 3 : 3 + d] = c.x
    c.x = big[:, 3 : 3 + d]
    logits = torch.zeros(t, 9, dtype=c.dt, device=DEV)
    logits[:, 2:6] = c.logits
    c.logits = logits[:, 2:6]
    wide = torch.zeros(4, 2 * f + 128, c.w1.shape[2] + 32, dtype=torch.uint8, device=DEV)
    wide[:, 128:, 16:-16] = c.w1.view(torch.uint8)
    c.w1 = wide[:, 128:, 16:-16].view(c.w1.dtype)
    scales = torch.zeros(4, c.w1_s.shape[1] + 2, *c.w1_s.shape[2:], dtype=torch.uint8, device=DEV)
    scales[:, 2:] = c.w1_s
    c.w1_s = scales[:, 2:]
    c.new()
    out = torch.full((t, d + 9), 7.0, dtype=c.dt, device=DEV)
    c.out = out[:, 5 : 5 + d]
    c.run()
    assert torch.equal(c.out, want)
    assert (out[:, :5] == 7.0).all() and (out[:, 5 + d :] == 7.0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_the_same_bits_every_time_and_on_another_stream(bits):
    c = Case(50, 8, 4, 640, 256, bits)
    want = c.run().clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        c.new()
        stream.wait_stream(torch.cuda.current_stream())
        c.run(stream)
        torch.cuda.current_stream().wait_stream(stream)
        assert torch.equal(c.out, want)


@pytest.mark.parametrize("bits", [8, 4])
def test_two_captured_calls_that_run_at_once(bits):
    """Two graphs on two streams, each with a workspace of its own, replayed on other inputs."""
    a, b = Case(3, 16, 4, 512, 256, bits, seed=3), Case(20, 8, 2, 384, 384, bits, seed=9)
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in (a, b):
        c.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    for c in (a, b):
        c.x.copy_(c.x.flip(0) * 1.5)
        c.logits.copy_(c.logits.flip(1))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_calls_behind_each_other_share_a_workspace():
    """A call's kernels start early: the next one's must not touch what this one still reads."""
    cases = [Case(t, 8, 2, 512, 256, 8, seed=t) for t in (1, 30, 2, 64)]
    room = max((c.workspace for c in cases), key=lambda w: w.numel())
    for c in cases:
        c.workspace = room
    for _ in range(10):
        for c in cases:
            c.run()
    for c in cases:
        c.check()


@pytest.mark.parametrize("bits", [8, 4])
def test_calls_that_feed_each_other_without_a_pause(bits):
    """A call's kernels begin before the ones before them have ended: inputs and weights that those are still writing."""
    e, d, f, k, t = 8, 256, 128, 2, 30
    layer, w = _layer(e, d, f, k, t, weight_bits=bits, training=False)
    logits = [torch.randn(t, e, device=DEV) for _ in range(12)]
    x0 = torch.randn(t, d, device=DEV).to(layer.dtype)
    weights = [w, (w.view(layer.dtype) * 1.5).view(torch.uint8)]

    def chain(pause):
        y, seen = x0, []
        for i, lg in enumerate(logits):
            if i % 3 == 0:
                layer.step(weights[i // 3 % 2])
                pause()
            y = layer.forward_tokens(y, lg)
            pause()
            y = layer.forward(y, lg) if i % 2 else y
            pause()
            y = (y / (y.abs().max() + 1e-3)).to(layer.dtype)
            seen.append(y)
        torch.cuda.synchronize()
        return seen

    want = chain(torch.cuda.synchronize)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(chain(lambda: None), want))
    layer.check_status()


def test_a_larger_workspace_and_a_status_word():
    from paper_2609_04609_b200 import ciera

    c = Case(5, 8, 2, 256, 128, 8)
    want = c.run().clone()
    room = torch.zeros(c.workspace.numel() + 4096, dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.zeros_like(c.out)
    ciera.expert_tokens(c.config, c.x, c.logits, c.bias, c.w1, c.w1_s, c.w2, c.w2_s, out, c.experts, c.weights, room, status)
    assert torch.equal(out, want) and int(status) == 0
    assert not room[: ciera.EXPERT_TOKENS_HEAD].any() and not room[-4096:].any()
    with pytest.raises(ciera.CieraError):
        ciera.expert_tokens(c.config, c.x, c.logits, c.bias, c.w1, c.w1_s, c.w2, c.w2_s, out, c.experts, c.weights, room[:512])


def test_no_tokens():
    c = Case(0, 8, 2, 128, 128, 8)
    c.run()


def _layer(e, d, f, k, t, dtype="bf16", **kw):
    from paper_2609_04609_b200 import runtime
    from paper_2609_04609_b200 import workloads as wl

    codec = runtime.LayerCodec.from_tensors([r * c for r, c in wl.olmoe_layer_shapes(e, d, f)], 4, dtype, 512, DEV)
    gen = wl.make_generator(5, DEV)
    w = wl.init_weights(codec.weights_bytes // wl.VALUE_BYTES[dtype], dtype, gen, d**-0.5)
    codec.init_caches(w.view(torch.uint8))
    return codec.expert_layer(e, d, f, k, t, **kw), w.view(torch.uint8)


def _off(y, want):
    return float((y.double() - want).norm() / want.norm())


def _want(layer, x, logits):
    at = layer.experts[: x.shape[0]].long()
    p = logits.double().softmax(1).gather(1, at)
    y = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    for e in range(layer.n_experts):
        t, j = (at == e).nonzero(as_tuple=True)
        h = torch.nn.functional.silu(x[t].double() @ layer.gate[e].double()) * (x[t].double() @ layer.up[e].double())
        y.index_add_(0, t, p[t, j, None] * (h @ layer.down[e].double()))
    return y


@pytest.mark.parametrize("bits,dtype,off_few,off_many", [
    # A weight rounded to e4m3 is off by 0.036 in the root of the mean square: the gate's and up's sums as well, silu(g) * u by
    # 0.036 * sqrt(2) * 1.25 = 0.064, the output by 0.073.  e2m1 has two bits less but keeps its steps above a group's small
    # values: off by 0.12 of a normal weight in the root of the mean square; 0.21 and 0.24.  With rounded rows as well sqrt(2) times that.
    (8, "bf16", 0.1, 0.15), (4, "bf16", 0.32, 0.45), (4, "fp16", 0.32, 0.45), (8, "fp32", 0.1, 0.15),
])
def test_layer_on_reconstructed_weights(bits, dtype, off_few, off_many):
    e, d, f, k, t = 8, 512, 256, 2, 100
    layer, w = _layer(e, d, f, k, t, dtype, weight_bits=bits, training=False)
    layer.step(w)
    x, logits = torch.randn(t, d, device=DEV).to(layer.dtype), torch.randn(t, e, device=DEV)
    y = layer.forward(x, logits)
    layer.check_status()
    assert _off(y, _want(layer, x, logits)) < off_many
    few = layer.forward_tokens(x[:20], logits[:20])
    assert _off(few, _want(layer, x[:20], logits[:20])) < off_few
    one = layer.forward_tokens(x[7:8], logits[7:8])
    assert torch.equal(one, few[7:8])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = layer.forward_tokens(x[:20], logits[:20], stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(other, few)
    with pytest.raises(ValueError):
        layer.forward_tokens(x[:65], logits[:65])


def test_layer_for_training_answers_too():
    e, d, f, k, t = 4, 256, 128, 2, 64
    layer, w = _layer(e, d, f, k, t)
    layer.step(w)
    x, logits = torch.randn(t, d, device=DEV).to(layer.dtype), torch.randn(t, e, device=DEV)
    layer.forward(x, logits)
    y = layer.forward_tokens(x, logits)
    assert _off(y, _want(layer, x, logits)) < 0.1
    with pytest.raises(RuntimeError):
        layer.backward(torch.ones_like(y))  # its choice has been written over
    layer.forward(x, logits)
    assert len(layer.backward(torch.ones_like(y))) == 5
    layer.check_status()
