"""How exactly the layer for a few tokens takes its values: sums of one term each, so that nothing but the parts of x and of silu(g) * u decides."""
import numpy as np
import pytest
import torch

from tests import parts_reference as pr
from tests.test_gpu_fp8 import DTYPES, E4M3
from tests.test_token_parts import EXACT, MANTISSA

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D, F, T = 384, 256, 20  # column 0 of x is the gate, alone in its 128; columns 128 on are the values


def _operand(w, bits):
    """w float32 [rows, cols] of powers of two and zeros, as a stack of one matrix; it has to be exact."""
    from paper_2609_04609_b200 import ciera

    rows, cols = w.shape
    w = w[None].to(DEV)
    back = torch.zeros_like(w)
    if bits == 8:
        q = torch.zeros(1, rows, cols, dtype=torch.uint8, device=DEV).view(E4M3)
        s = torch.zeros(1, -(-rows // 128), cols // 128, dtype=torch.uint8, device=DEV)
        ciera.fp8_quantize_blocks(w, q, s)
        back = q.float() * torch.exp2(s.float() - 127).repeat_interleave(128, 1).repeat_interleave(128, 2)
    else:
        q = torch.zeros(1, rows, cols // 2, dtype=torch.uint8, device=DEV)
        s = torch.full((1, -(-rows // 128), cols // 128, 512), 127, dtype=torch.uint8, device=DEV)
        ciera.fp4_quantize_matrices(w, q, s)
        ciera.fp4_values(q, s, back)
    assert torch.equal(back, w)
    return q, s


def _pick(values, dtype, bits, x_order, h_order):
    """values [T, F] through the layer: value i is x's column 128 + x_order[i] and column h_order[i] of the middle, 64 times as large;
    out[:, i] is the middle's value i again."""
    from paper_2609_04609_b200 import ciera

    t = values.shape[0]
    x = torch.zeros(t, D, dtype=torch.float64)
    x[:, 0] = 1.0
    x[:, 128 + x_order] = torch.from_numpy(values)
    x = x.to(DTYPES[dtype])
    w1 = torch.zeros(2 * F, D)
    w1[:F, 0] = 64.0
    w1[F + h_order, 128 + x_order] = 1.0
    w2 = torch.zeros(D, F)
    w2[torch.arange(F), h_order] = 1.0
    w1, w1_s = _operand(w1, bits)
    w2, w2_s = _operand(w2, bits)
    config = ciera.RouteConfig(n_experts=1, top_k=1, n_groups=1, top_groups=1, group_best=1, score=ciera.SCORE_SOFTMAX, renormalise=0, scale=1.0)
    out = torch.zeros(t, D, dtype=DTYPES[dtype], device=DEV)
    experts, weights = torch.zeros(t, 1, dtype=torch.int32, device=DEV), torch.zeros(t, 1, device=DEV)
    workspace = torch.zeros(ciera.expert_tokens_workspace_bytes(config, t, D, F), dtype=torch.uint8, device=DEV)
    ciera.expert_tokens(config, x.to(DEV), torch.zeros(t, 1, device=DEV), None, w1, w1_s, w2, w2_s, out, experts, weights, workspace)
    assert (weights == 1.0).all() and (out[:, F:] == 0).all()
    return out[:, :F].double().cpu().numpy() / 64


def _orders(how):
    """Places of values 0 ... F - 1, of which every 32nd is a large one: beside the others ("both"), or all in groups of their own in x, in
    the middle, or in neither of the two."""
    here, i = torch.arange(F), torch.arange(F)
    large = i % 32 == 0
    apart = torch.empty(F, dtype=torch.long)
    apart[large] = torch.arange(int(large.sum()))
    # the large ones' group is filled up by values that the test leaves alone
    apart[~large] = torch.arange(int(large.sum()), F)
    return {"both": (here, here), "x": (here, apart), "middle": (apart, here)}[how]


def _values(ratio, mantissa, seed, dtype, large):
    """[T, F]: every 32nd `large`, the rest `ratio` powers of two below it."""
    g = np.random.default_rng(seed)
    v = large * 2.0**-ratio * (1 + np.floor(g.random((T, F)) * 2.0**mantissa) * 2.0**-mantissa) * g.choice([-1.0, 1.0], (T, F))
    v[:, ::32] = large * (1 + np.floor(g.random((T, F // 32)) * 2.0**mantissa) * 2.0**-mantissa)
    return torch.from_numpy(v).to(DTYPES[dtype]).double().numpy()


def _grouped(values, order):
    at = np.zeros_like(values)
    at[:, order.numpy()] = values
    return at


@pytest.mark.parametrize("how", ["both", "x", "middle"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("bits", [8, 4])
def test_values_of_16_bits_beside_larger_ones_are_exact(bits, dtype, how):
    """The large ones are at most twice 2^(ratio) times as large, so ratio is one less than what is stated."""
    ratio = EXACT[bits][dtype] - 1
    v = _values(ratio, MANTISSA[dtype], ratio, dtype, 256.0)
    orders = _orders(how)
    for order in orders:
        assert np.array_equal(pr.split(_grouped(v, order), bits, pr.PARTS[bits][2]), _grouped(v, order))
    fewer = [_grouped(v, o) - pr.split(_grouped(v, o), bits, pr.PARTS[bits][2] - 1) for o in orders]
    assert max(np.abs(f).max() for f in fewer) > 0.1 * 2.0**-ratio * 256.0 * 2.0 ** -MANTISSA[dtype]  # one part less would be seen
    assert np.array_equal(_pick(v, dtype, bits, *orders), v)


@pytest.mark.parametrize("how", ["both", "x", "middle"])
@pytest.mark.parametrize("bits,ratio", [(8, 0), (8, 6), (8, 26), (4, 10), (4, 14)])
def test_values_of_32_bits(bits, ratio, how):
    """Both splits leave out what they may at most; the parts are added up in 32 bits, small ones first (their sums are at most the value
    and what is left of the largest: a step of each, twice two values' worth)."""
    v = _values(ratio, 23, 5 + ratio, "fp32", 256.0)
    parts = pr.PARTS[bits][4]
    orders = _orders(how)
    tol, fewer = np.zeros_like(v), np.zeros_like(v)
    for order in orders:
        at = _grouped(v, order)
        tol += pr.bound(at, bits, parts)[:, order.numpy()]
        fewer = np.maximum(fewer, np.abs(pr.split(at, bits, parts - 1) - at)[:, order.numpy()])
    tol += 4 * 2.0**-24 * np.abs(v)
    small = np.arange(F) % 32 != 0
    assert (fewer[:, small] > tol[:, small]).any()  # one part less would be seen
    off = np.abs(_pick(v, "fp32", bits, *orders) - v)[:, small]
    assert (off <= tol[:, small]).all(), float((off / tol[:, small]).max())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_many_terms_in_the_root_of_the_mean_square(bits, dtype):
    """Ordinary values through ordinary weights, with one value 64 times the rest in each 32: off by no more than the rounding of the result
    and the root of the number of terms times a step of 32 bits, where what the parts leave out is counted as it falls (spread evenly,
    0.29 of what is left out at most, which is counted whole)."""
    from tests.test_gpu_expert_tokens import Case

    c = Case(24, 2, 1, 512, 256, bits, dtype, seed=11)
    c.x[:, ::32] *= 64
    c.x = (c.x * 2.0**-3).contiguous()
    c.run()
    out, size = torch.zeros(24, 512, dtype=torch.float64, device=DEV), torch.zeros(24, 512, dtype=torch.float64, device=DEV)
    left = torch.zeros_like(out)
    x = c.x.double()
    parts = pr.PARTS[bits][4 if dtype == "fp32" else 2]
    x_left = torch.from_numpy(pr.bound(x.cpu().numpy(), bits, parts)).to(DEV)
    for e in range(2):
        t = (c.experts[:, 0] == e).nonzero()[:, 0]
        w = c.weights[t].double()
        v1, v2 = c.v1[e], c.v2[e]
        h = x[t] @ v1.T
        gate, up = h[:, :256], h[:, 256:]
        sig = torch.sigmoid(gate)
        a = gate * sig * up
        slope = sig * (1 + gate * (1 - sig))
        # squares: what each term is off by
        term = (2.0**-23 * 4) ** 2  # sums of parts and of terms, silu to 2^-21 of itself
        h2 = (x_left[t] ** 2) @ (v1**2).T + term * ((x[t] ** 2) @ (v1**2).T)
        a2 = (slope * up) ** 2 * h2[:, :256] + (gate * sig) ** 2 * h2[:, 256:] + term * a**2
        a_left = torch.from_numpy(pr.bound(a.cpu().numpy(), bits, parts)).to(DEV)
        out[t] = w * (a @ v2.T)
        left[t] = w**2 * ((a2 + a_left**2 + term * a**2) @ (v2**2).T)
    step = torch.finfo(c.dt).eps / 2
    want = float((left + (step * out) ** 2).mean().sqrt())
    off = float((c.out.double() - out).square().mean().sqrt())
    assert off <= want, off / want
