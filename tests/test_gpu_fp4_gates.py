"""silu(g) * u in 4 bits where a factor is at the end of its range."""
import numpy as np
import pytest
import torch

from tests import fp4_reference as f4
from tests import moe_reference as ref
from tests.test_gpu_fp8 import DTYPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(x, cols):
    from paper_2609_04609_b200 import ciera

    rows = x.shape[0]
    q = torch.zeros(rows, -(-cols // 32) * 16, dtype=torch.uint8, device=DEV)[:, : (cols + 1) // 2]
    atoms = torch.zeros(-(-rows // 128), -(-cols // 128), 512, dtype=torch.uint8, device=DEV)
    ciera.fp4_quantize_rows(x.to(DEV), q, atoms, kind=ciera.SOURCE_SWIGLU)
    want = ref.swiglu(x.double().numpy())
    _, s = f4.quantize(want)
    assert np.array_equal(f4.scale_bytes(atoms, rows, cols), s)
    # off by at most 20 steps of 32 bits before the rounding, half a step of which is at most 1/4 of the value or of the scale
    unit = np.repeat(2.0 ** (s - 127.0), 32, 1)[:, :cols]
    have = f4.values(f4.unpack(q, cols), s)
    off = np.abs(have - want) - np.maximum(np.abs(want) / 4, unit / 4) * (1 + 2.0**-18)
    assert (off <= 0).all(), float(off.max())


@pytest.mark.parametrize("cols", [64, 33])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_tiny_gates_beside_huge_ups(dtype, cols):
    """Gates of few bits (below 2^-126), whose silu has a bit less: ups so large that the product is an ordinary number."""
    g = torch.Generator().manual_seed(3)
    gate = torch.randn(40, cols, generator=g) * torch.exp2(-torch.randint(100, 149, (40, cols), generator=g).float())
    gate[0], gate[1] = 2.0**-149 * (4096 if dtype == "bf16" else 1), 2.0**-133 * 3
    up = torch.randn(40, cols, generator=g) * 2.0**100
    up[0], up[1] = 2.0**127, 1.75 * 2.0**126
    x = torch.cat([gate, up], 1).to(DTYPES[dtype])
    assert ((x[:, :cols] != 0) & (x[:, :cols].abs() < 2.0**-126)).any()
    _check(x, cols)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_huge_gates_and_gates_far_below_zero(dtype):
    g = torch.Generator().manual_seed(4)
    gate = torch.randn(40, 64, generator=g) * torch.exp2(torch.randint(-10, 100, (40, 64), generator=g).float())
    gate[:20] = -torch.rand(20, 64, generator=g) * 86.5
    up = torch.randn(40, 64, generator=g) * torch.exp2(torch.randint(-120, 20, (40, 64), generator=g).float())
    up[:10] *= 2.0**100
    _check(torch.cat([gate, up], 1).to(DTYPES[dtype]), 64)
