"""Routing of tokens to experts and its gradient against 64-bit arithmetic."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _config(E, k, score, G=1, top_groups=1, best=2, renorm=False, scale=1.0):
    from paper_2609_04609_b200 import ciera

    code = {"softmax": ciera.SCORE_SOFTMAX, "sigmoid": ciera.SCORE_SIGMOID}[score]
    return ciera.RouteConfig(n_experts=E, top_k=k, n_groups=G, top_groups=top_groups, group_best=best, score=code,
                             renormalise=int(renorm), scale=scale)


def _logits(T, E, dtype, seed, std=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * std).to(DTYPES[dtype])


def _check(logits, bias, E, k, score, G=1, top_groups=1, best=2, renorm=False, scale=1.0, strided=False):
    from paper_2609_04609_b200 import ciera

    T = logits.shape[0]
    dev = logits.to(DEV)
    if strided:
        dev = torch.cat([dev, torch.full((T, 3), 9.0, dtype=dev.dtype, device=DEV)], 1)[:, :E]
    experts = torch.full((T + 1, k), -7, dtype=torch.int32, device=DEV)
    weights = torch.full((T + 1, k), -7.0, device=DEV)
    ciera.route(_config(E, k, score, G, top_groups, best, renorm, scale), dev, None if bias is None else bias.to(DEV),
                experts[:T], weights[:T])
    torch.cuda.synchronize()
    ids, w = ref.route(logits, bias, k, score, G, top_groups, best, renorm, scale)
    assert np.array_equal(experts[:T].cpu().numpy(), ids)
    assert (experts[T] == -7).all() and (weights[T] == -7).all()
    # a weight is a quotient of sums of at most E terms in 32 bits: each term is off by a few steps, each addition by half of one
    tol = (E + 16) * 2.0**-24 * np.abs(w) + 1e-37
    assert (np.abs(weights[:T].cpu().numpy() - w) <= tol).all()
    # the same tokens over and over in a batch that is done several tokens a warp
    n = -(-4801 // T)
    many_e = torch.full((n * T, k), -7, dtype=torch.int32, device=DEV)
    many_w = torch.full((n * T, k), -7.0, device=DEV)
    ciera.route(_config(E, k, score, G, top_groups, best, renorm, scale), dev.repeat(n, 1), None if bias is None else bias.to(DEV),
                many_e, many_w)
    many_e, many_w = many_e.view(n, T, k).cpu().numpy(), many_w.view(n, T, k).cpu().numpy()
    assert (many_e == ids).all() and (np.abs(many_w - w) <= tol).all()
    return experts[:T], weights[:T]


@pytest.mark.parametrize("T,E,k,score,G,top_groups,best,bias,renorm,scale,dtype", [
    (1, 64, 8, "softmax", 1, 1, 2, False, False, 1.0, "bf16"),
    (1, 1, 1, "softmax", 1, 1, 1, False, True, 1.0, "fp32"),
    (7, 8, 2, "softmax", 1, 1, 2, False, True, 1.0, "fp32"),
    (129, 60, 4, "softmax", 1, 1, 2, True, False, 1.0, "fp16"),
    (300, 256, 8, "sigmoid", 8, 4, 2, True, True, 2.5, "bf16"),
    (300, 160, 6, "softmax", 8, 3, 1, False, False, 16.0, "bf16"),
    (65, 96, 32, "sigmoid", 32, 31, 2, True, True, 1.0, "fp32"),
    (33, 33, 11, "sigmoid", 3, 1, 2, False, False, 1.0, "fp16"),
    (40, 384, 8, "sigmoid", 1, 1, 2, True, True, 2.5, "fp32"),
    (20, 1024, 32, "softmax", 4, 2, 2, True, True, 1.0, "bf16"),
    (20, 1000, 10, "sigmoid", 1, 1, 2, True, False, 1.0, "bf16"),
    (6000, 64, 8, "softmax", 1, 1, 2, False, False, 1.0, "bf16"),
])
def test_route_equals_64_bit_arithmetic(T, E, k, score, G, top_groups, best, bias, renorm, scale, dtype):
    b = (torch.rand(E, generator=torch.Generator().manual_seed(3)) - 0.5) * 0.2 if bias else None
    for strided in (False, True):
        _check(_logits(T, E, dtype, 11 + T), b, E, k, score, G, top_groups, best, renorm, scale, strided)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,top_groups", [(1, 1), (4, 2)])
def test_equal_scores_go_to_the_lower_index(score, G, top_groups):
    coarse = torch.randint(-2, 3, (200, 64), generator=torch.Generator().manual_seed(1)).float()
    coarse[0] = 0.0
    coarse[1] = 50.0  # sigmoid: equal in 64 bits although the logits differ
    coarse[1, 40:] = 51.0
    for bias in (None, torch.zeros(64), torch.randint(0, 2, (64,), generator=torch.Generator().manual_seed(2)).float() * 0.25):
        _check(coarse, bias, 64, 6, score, G, top_groups, 2, True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_next_to_each_other_are_told_apart(score):
    """c of two experts differs by less than a step of 32 bits: the choice is that of 64."""
    E = 64
    logits = _logits(500, E, "fp32", 5)
    s, _ = ref.scores(logits, score)
    bias = torch.zeros(E)
    # expert 1 gets expert 0's logit moved by one to three steps of 32 bits, in either direction
    for t in range(500):
        x = np.float32(3.0 + 0.001 * t)
        y = x
        for _ in range(1 + t % 3):
            y = np.nextafter(y, np.float32(9.0 if t % 2 else -9.0))
        logits[t, 0], logits[t, 1] = float(x), float(y)
    _check(logits, None, E, 4, score)
    bias[0] = 1e-3
    _check(logits, bias, E, 4, score, 8, 3, 2, True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,top_groups", [(1, 1), (8, 3)])
def test_closed_experts_and_special_values(score, G, top_groups):
    E, k = 64, 8
    x = _logits(64, E, "fp32", 8)
    x[0] = float("-inf")  # nothing left
    x[1] = float("nan")
    x[2, 5:] = float("-inf")  # fewer than k left
    x[3, ::2] = float("nan")
    x[4] = torch.finfo(torch.float32).min  # a mask of the lowest value: all equal
    x[5, 7] = float("inf")
    x[6, 7], x[6, 9] = float("inf"), float("inf")
    x[7, : E // 2] = torch.finfo(torch.float32).min
    x[8, :56] = float("-inf")  # one group of eight left
    bias = (torch.rand(E, generator=torch.Generator().manual_seed(3)) - 0.5) * 0.2
    bias[11], bias[12], bias[13] = float("-inf"), float("nan"), float("inf")
    for b in (None, bias):
        for renorm in (False, True):
            ids, w = _check(x, b, E, k, score, G, top_groups, 2, renorm, 1.5)
            assert (ids[:2] == -1).all() and (w[:2] == 0).all()
    for dt in ("bf16", "fp16"):
        y = x.clone()
        y[4] = torch.finfo(DTYPES[dt]).min
        y[7, : E // 2] = torch.finfo(DTYPES[dt]).min
        _check(y.to(DTYPES[dt]), bias, E, k, score, G, top_groups, 2, True)


@pytest.mark.parametrize("T,E,k,score,renorm,dtype", [
    (1, 64, 8, "softmax", False, "bf16"), (1, 1, 1, "sigmoid", False, "fp32"), (130, 60, 4, "softmax", True, "fp16"),
    (300, 256, 8, "sigmoid", True, "bf16"), (70, 100, 3, "sigmoid", False, "fp32"), (50, 1024, 32, "softmax", False, "fp32"),
    (3000, 64, 8, "softmax", True, "fp32"),
])
def test_route_backward_equals_the_formula(T, E, k, score, renorm, dtype):
    from paper_2609_04609_b200 import ciera

    logits = _logits(T, E, dtype, 21 + T)
    logits[T // 2, : E // 2] = float("-inf")
    if T > 3:
        logits[3] = float("-inf")
    ids, _ = ref.route(logits, None, k, score)
    experts = torch.from_numpy(ids).to(torch.int32)
    if T > 5 and k > 2:
        experts[4, 1] = E  # outside: passed over
        experts[5, 0] = experts[5, 2]  # the same index twice
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(4))
    dw[experts < 0] = 1e30  # passed over too
    want = ref.route_backward(logits, experts, dw, score, renorm, 2.0)
    wide = torch.full((T, E + 3), 7.0, dtype=DTYPES[dtype], device=DEV)
    out = wide[:, :E]
    ciera.route_backward(_config(E, k, score, renorm=renorm, scale=2.0), logits.to(DEV), experts.to(DEV), dw.to(DEV), out)
    torch.cuda.synchronize()
    assert (wide[:, E:] == 7.0).all()
    # dl = s (ds - dot): s is off by (E + 8) steps of 32 bits, ds and dot by at most (E + k + 16) steps of the largest term, and the
    # result is rounded to its type
    s, _ = ref.scores(logits, score)
    some = (ids >= 0)
    d = np.where(some, np.abs(dw.numpy().astype(np.float64)), 0.0)
    d[d > 1e29] = 0.0
    term = 2.0 * d.max(1, initial=0.0)
    if renorm:
        total = np.array([sum(s[t, e] for e in experts[t].tolist() if 0 <= e < E) for t in range(T)])
        term = np.where(total > 0, 2 * term / np.where(total > 0, total, 1), 0.0)
    step = torch.finfo(DTYPES[dtype]).eps / 2
    tol = 2 * (E + k + 24) * 2.0**-24 * s * term[:, None] * (k + 1) + step * np.abs(want) + 6e-8 * (dtype == "fp16") + 1e-37
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_backward_equals_differences(score, renorm):
    """The loss sum(dw * w) of 64-bit weights, moved by 1e-6 in every logit, while the choice stays."""
    from paper_2609_04609_b200 import ciera

    T, E, k = 3, 12, 4
    logits = _logits(T, E, "fp32", 77)
    ids, _ = ref.route(logits, None, k, score)
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(6))

    def loss(x):
        s, _ = ref.scores(x, score)
        w = np.take_along_axis(s, ids, 1)
        w = w / w.sum(1, keepdims=True) if renorm else w
        return (w * 1.5 * dw.double().numpy()).sum(1)

    out = torch.zeros(T, E, device=DEV)
    ciera.route_backward(_config(E, k, score, renorm=renorm, scale=1.5), logits.to(DEV),
                         torch.from_numpy(ids).to(torch.int32).to(DEV), dw.to(DEV), out)
    got = out.cpu().numpy()
    for e in range(E):
        h = torch.zeros(T, E, dtype=torch.float64)
        h[:, e] = 1e-6
        diff = (loss(logits.double() + h) - loss(logits.double() - h)) / 2e-6
        # the differences' own error: third derivatives (below 10) times h^2, 64-bit rounding over h
        assert np.allclose(got[:, e], diff, rtol=2e-5, atol=1e-6)


def test_route_on_another_stream_and_in_a_graph():
    from paper_2609_04609_b200 import ciera

    T, E, k = 100, 64, 8
    cfg = _config(E, k, "sigmoid", 8, 4, 2, True, 2.5)
    bias = torch.zeros(E, device=DEV)
    x = _logits(T, E, "bf16", 1).to(DEV)
    experts = torch.zeros(T, k, dtype=torch.int32, device=DEV)
    weights = torch.zeros(T, k, device=DEV)
    dw = torch.ones(T, k, device=DEV)
    dl = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ciera.route(cfg, x, bias, experts, weights)
        ciera.route_backward(cfg, x, experts, dw, dl)
    graph = torch.cuda.CUDAGraph()
    side.synchronize()
    with torch.cuda.graph(graph):
        ciera.route(cfg, x, bias, experts, weights)
        ciera.route_backward(cfg, x, experts, dw, dl)
    for seed in (2, 3):
        new = _logits(T, E, "bf16", seed)
        x.copy_(new)
        bias.copy_(torch.rand(E, generator=torch.Generator().manual_seed(seed)) * 0.1)
        graph.replay()
        torch.cuda.synchronize()
        ids, w = ref.route(new, bias.cpu(), k, "sigmoid", 8, 4, 2, True, 2.5)
        assert np.array_equal(experts.cpu().numpy(), ids)
        want = ref.route_backward(new, experts, dw, "sigmoid", True, 2.5)
        assert np.abs(dl.double().cpu().numpy() - want).max() <= 2.0**-8 * np.abs(want).max() + 1e-5
    ciera.route(cfg, x[:0], bias, experts[:0], weights[:0])  # no tokens
    ciera.route_backward(cfg, x[:0], experts[:0], dw[:0], dl[:0])
