"""Routing where 32 bits and 64 part: zeros of either sign, neighbours that the lists do not hold, sums that overflow or vanish."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref
from tests.test_gpu_route import DEV, DTYPES, _check, _config, _logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_zeros_of_either_sign_are_equal(score, dtype):
    g = torch.Generator().manual_seed(1)
    for E, k in ((2, 1), (64, 6), (200, 8)):
        x = torch.where(torch.rand(100, E, generator=g) < 0.5, torch.tensor(0.0), torch.tensor(-0.0))
        x[50:] = torch.where(torch.rand(50, E, generator=g) < 0.7, -torch.rand(50, E, generator=g), x[50:])
        x = x.to(DTYPES[dtype])
        assert bool(torch.signbit(x[:50]).any()) and not bool(torch.signbit(x[:50]).all())
        _check(x, None, E, k, score)
        _check(x, torch.zeros(E), E, k, score, 2, 1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [64, 256, 1000])
def test_equal_scores_hide_no_larger_one(score, E):
    """k + 1 and more equal logits at low places, and one that is larger by a step or a few of 32 bits at a high one."""
    g = torch.Generator().manual_seed(E)
    for k in (1, 3, 8):
        x = torch.randn(60, E, generator=g)
        for t in range(60):
            low = torch.randperm(E // 2, generator=g)[: k + 1 + t % 3]
            x[t, low] = 6.0
            y = np.float32(6.0)
            for _ in range(1 + t % 31):
                y = np.nextafter(y, np.float32(9))
            x[t, E // 2 + t % (E // 2)] = float(y)
        ids, _ = _check(x, None, E, k, score)
        assert (ids[:, 0].cpu() == E // 2 + torch.arange(60) % (E // 2)).all()
        _check(x, torch.zeros(E), E, k, score)
        _check(x, torch.zeros(E), E, k, score, 2, 2)


@pytest.mark.parametrize("E", [8, 64, 100])
@pytest.mark.parametrize("G,top_groups", [(1, 1), (4, 3)])
def test_a_large_score_with_a_bias_against_it(E, G, top_groups):
    """c of a large score and a large negative bias beside c of a small score: the error of the large one counts."""
    rng = np.random.default_rng(E)
    T = 500
    x = rng.standard_normal((T, E)).astype(np.float32)
    bias = torch.zeros(E)
    b0 = float(np.float32(-0.98))
    bias[0] = b0
    x[:, 1] = np.abs(x[:, 1]) + 2.0
    for t in range(T):  # s0 + b0 = s1, solved for the first logit, and a few steps to either side
        e = np.exp(x[t].astype(np.float64))
        rest = e[1:].sum()
        y = np.float32(np.log((-b0 * rest + e[1]) / (1 + b0)))
        for _ in range(t % 4):
            y = np.nextafter(y, np.float32(90.0 if t % 8 < 4 else -90.0))
        x[t, 0] = y
    logits = torch.from_numpy(x)
    s, _ = ref.scores(logits, "softmax")
    assert (np.abs(s[:, 0] + b0 - s[:, 1]) < 1e-7).all()
    for k in (1, 2, 5):
        if k <= top_groups * (E // G):
            _check(logits, bias, E, k, "softmax", G, top_groups, 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best", [1, 2])
def test_a_bias_of_the_lowest_value_closes_nothing(score, best):
    E, G = 16, 4
    x = _logits(80, E, "fp32", 3)
    x[5, 4:8] = float("-inf")
    bias = torch.full((E,), torch.finfo(torch.float32).min)
    bias[8:12] = 0.0
    for k, top_groups in ((6, 2), (4, 1), (12, 3)):
        ids, _ = _check(x, bias, E, k, score, G, top_groups, best, True)
        assert (ids >= 0).all()
    bias[8:12] = torch.finfo(torch.float32).min
    _check(x, bias, E, 6, score, G, 2, best)


def _small_scores(score, T=120, E=32):
    """Logits, a bias under which only small scores are chosen, and how many bits below 1 those lie."""
    g = torch.Generator().manual_seed(9)
    x = _logits(T, E, "fp32", 31)
    depth = torch.linspace(60.0, 690.0, T)[:, None]
    if score == "sigmoid":
        return x - depth, None
    x[:, 1:] -= depth  # the first takes all of the softmax, and the bias keeps it from being chosen
    x[:, 0] = 0.0
    bias = torch.zeros(E)
    bias[0] = -5.0
    bias[1:] = torch.rand(E - 1, generator=g)
    return x, bias


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_weights_of_scores_that_vanish_in_32_bits_are_quotients(score):
    x, bias = _small_scores(score)
    _, w = _check(x, bias, 32, 4, score, renorm=True, scale=2.5)
    total = w.sum(1).cpu()
    assert ((total - 2.5).abs() < 1e-5).all()
    _check(x, bias, 32, 4, score, 4, 2, 2, renorm=True)
    far = x.clone()
    far[:60, 1:] -= 1e6  # vanish in 64 bits as well: the sum is 0
    far[:60, 0] -= 1e6 if score == "sigmoid" else 0.0
    _check(far, bias, 32, 4, score, renorm=True)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [32, 200])
def test_gradients_through_scores_that_vanish_in_32_bits(score, E):
    from paper_2609_04609_b200 import ciera

    x, bias = _small_scores(score, 110, E)
    x = torch.cat([x[:100], x[:100] - 1e6])
    if score == "softmax":
        x[100:, 0] = 0.0
    k = 4
    ids, w = ref.route(x, bias, k, score, renormalise=True)
    dw = torch.randn(200, k, generator=torch.Generator().manual_seed(4))
    ids[7, 1] = ids[7, 0]  # the same index twice
    ids[8, 2] = -1
    experts = torch.from_numpy(ids).to(torch.int32)
    want = ref.route_backward(x, experts, dw, score, True, 2.0)
    assert np.isfinite(want).all() and (want[100:] == 0).all() and (np.abs(want[:100]).max(1) > 0).all() and np.abs(want).max() > 0.1
    out = torch.full((200, E), 7.0, device=DEV)
    ciera.route_backward(_config(E, k, score, renorm=True, scale=2.0), x.to(DEV), experts.to(DEV), dw.to(DEV), out)
    # dl = p (d - sum of p d) for p, d of the chosen: a product and a difference of numbers up to 2 max |d|, each off by a few steps
    # (quotients, at most k terms), beside a factor 1 - s
    tol = (k + 24) * 2.0**-24 * 4.0 * 2 * dw.abs().max().item() + 1e-37
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


def test_every_number_of_tokens_around_the_change_of_kernels():
    """From one warp a token to several tokens a warp: the last of them alone in its warp, and in its block."""
    E, k = 64, 4
    from paper_2609_04609_b200 import ciera

    x = _logits(4800, E, "bf16", 2)
    ids, w = ref.route(x, None, k, "softmax")
    dev = x.to(DEV)
    for T in (4735, 4736, 4737, 4743, 4744, 4745, 4767, 4768, 4769):
        experts = torch.full((T + 1, k), -7, dtype=torch.int32, device=DEV)
        weights = torch.full((T + 1, k), -7.0, device=DEV)
        ciera.route(_config(E, k, "softmax"), dev[:T], None, experts[:T], weights[:T])
        assert np.array_equal(experts[:T].cpu().numpy(), ids[:T])
        assert np.allclose(weights[:T].cpu().numpy(), w[:T], rtol=(E + 16) * 2.0**-24, atol=0)
        assert (experts[T] == -7).all() and (weights[T] == -7).all()
