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
