"""The end of a call of the layer for a few tokens: counters are zero behind it, and one that is given up is followed by none that goes by
its counters."""
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


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place(bits, dtype):
    """The output is written when every block has read what it needs of x."""
    c = Case(50, 8, 4, 640, 256, bits, dtype)
    _call(c, None)
    want, x = c.out.clone(), c.x.clone()
    for _ in range(20):
        c.x.copy_(x)
        c.out = c.x
        _call(c, None)
        assert torch.equal(c.out, want)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("counter", [0, 2])
def test_a_wait_that_runs_out_is_reported_until_the_workspace_is_zeros_again(bits, counter):
    """A counter that starts one below zero never gets to the number of blocks: the bounded wait for parts (0) or for all tiles (2) runs out
    after a second or two, the kernel comes back by itself, and nothing is written."""
    from paper_2609_04609_b200 import ciera

    c = Case(5, 16, 4, 512, 256, bits)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    words = c.workspace[: ciera.EXPERT_TOKENS_HEAD].view(torch.int32)
    words[counter] = -1
    _call(c, status)
    torch.cuda.synchronize()
    assert int(status) == ciera.ERR_TIMEOUT and (c.out == 7.0).all()
    for _ in range(2):  # whatever the counters are now
        status.zero_()
        _call(c, status)
        torch.cuda.synchronize()
        assert int(status) == ciera.ERR_TIMEOUT and (c.out == 7.0).all()
    _call(c, None)  # nobody is told, and nothing written either
    assert (c.out == 7.0).all()
    status.zero_()
    words.zero_()
    _call(c, status)
    assert int(status) == 0
    c.check()


def test_a_layer_that_gave_up_is_usable_again():
    from paper_2609_04609_b200 import ciera

    from tests.test_gpu_expert_tokens import _layer

    e, d, f, k, t = 8, 256, 128, 2, 16
    layer, w = _layer(e, d, f, k, t, weight_bits=4, training=False)
    layer.step(w)
    x, logits = torch.randn(t, d, device=DEV).to(layer.dtype), torch.randn(t, e, device=DEV)
    want = layer.forward_tokens(x, logits)
    layer.check_status()
    layer.few_workspace.view(torch.int32)[0] = -(1 << 31)  # as a call that was given up leaves it
    out = layer.forward_tokens(x, logits, out=torch.full_like(x, 7.0))
    with pytest.raises(ciera.CieraError) as error:
        layer.check_status()
    assert error.value.status == ciera.ERR_TIMEOUT and (out == 7.0).all()
    assert torch.equal(layer.forward_tokens(x, logits), want)
    layer.check_status()
