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
