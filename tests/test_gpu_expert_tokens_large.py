"""The layer for a few tokens at the ends of its range of widths, against 64 bits."""
import pytest
import torch

from tests.test_gpu_expert_tokens import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("t,e,k,d,f,dtype", [
    (1, 2, 1, 65536, 128, "bf16"), (3, 2, 2, 128, 65536, "bf16"), (20, 1, 1, 65536, 256, "fp32"), (64, 2, 1, 256, 65536, "fp16"),
    (33, 3, 2, 16384, 640, "bf16"),
])
def test_widest(t, e, k, d, f, dtype, bits):
    c = Case(t, e, k, d, f, bits, dtype)
    if dtype == "fp16":
        c.x *= 2.0**-4  # (the output of so wide a layer would leave fp16)
    c.run()
    assert torch.isfinite(c.out).all()
    c.check()
