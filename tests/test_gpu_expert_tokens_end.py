"""The end of a call of the layer for a few tokens: counters are zero behind it."""
import pytest
import torch

from tests.test_gpu_expert_tokens import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _call(c, status):
    from paper_2609_04609_b200 import ciera

    ciera.expert_tokens(c.config, c.x, c.logits, c.bias, c.w1, c.w1_s, c.w2, c.w2_s, c.out, c.experts, c.weights, c.workspace, status)


@pytest.mark.parametrize("bits,t,e,k,d,f", [(8, 1, 16, 8, 512, 128), (8, 40, 16, 4, 1024, 256), (4, 64, 32, 8, 2048, 256), (4, 5, 256, 8, 1024, 512),
                                            (8, 64, 4, 2, 128, 384)])
def test_counters_are_zero_behind_calls_whose_tiles_some_warps_have_no_part_in(bits, t, e, k, d, f):
    """A tile of fewer than four stages leaves column warps that only wait for its group; calls behind each other on one workspace."""
    from paper_2609_04609_b200 import ciera

    c = Case(t, e, k, d, f, bits)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    _call(c, status)
    want = c.out.clone()
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(300):
        c.out.fill_(7.0)
        _call(c, status)
        bad += c.workspace[: ciera.EXPERT_TOKENS_HEAD].ne(0).sum() + c.out.ne(want).sum()
    assert int(bad) == 0 and int(status) == 0
    c.check()
