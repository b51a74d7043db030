"""The MoE layer on a stream of its own: where its results and inputs live, and what a refused call leaves."""
import pytest
import torch

from paper_2609_04609_b200 import workloads as wl
from tests.test_gpu_expert_layer import DEV, _layer

pytestmark = pytest.mark.gpu


def _inputs(layer, t, seed):
    gen = wl.make_generator(seed, DEV)
    x = torch.randn(t, layer.d_model, generator=gen, device=DEV).to(layer.dtype)
    logits = torch.randn(t, layer.n_experts, generator=gen, device=DEV)
    return x, logits, torch.randn(t, layer.d_model, generator=gen, device=DEV).to(layer.dtype)


def test_results_of_a_side_stream_are_not_memory_that_the_current_one_still_uses():
    e, d, f, k, t = 8, 256, 128, 2, 512
    layer, w = _layer(e, d, f, k, t)
    layer.step(w)
    x, logits, dout = _inputs(layer, t, 3)
    want = (layer.forward(x, logits),) + layer.backward(dout)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        # memory of the results' sizes, written late on the current stream and already given back to its pool
        torch.cuda._sleep(20_000_000)
        late = [torch.empty_like(r) for r in want]
        for r in late:
            r.fill_(7.0)
        del late
        got = (layer.forward(x, logits, stream=side),) + layer.backward(dout, stream=side)
        torch.cuda.synchronize()
        layer.check_status()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got


def test_inputs_and_results_that_are_dropped_early_stay_until_the_stream_is_done():
    e, d, f, k, t = 8, 256, 128, 2, 512
    layer, w = _layer(e, d, f, k, t)
    layer.step(w)
    x, logits, dout = _inputs(layer, t, 4)
    want = (layer.forward(x, logits),) + layer.backward(dout)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        mine = [v.clone() for v in (x, logits, dout)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        y = layer.forward(mine[0], mine[1], stream=side)
        got = (y,) + layer.backward(mine[2], stream=side)
        shapes = [(v.shape, v.dtype) for v in mine]
        layer.forward(x[:0], logits[:0])  # the layer lets go of the batch
        del mine, y
        for shape, dtype in shapes * 2:  # the current stream takes such memory and writes it at once
            torch.full(shape, 9.0, dtype=dtype, device=DEV)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_tokens_on_a_side_stream():
    layer, w = _layer(4, 128, 128, 2, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer.step(w, stream=side)
    y = layer.forward(torch.zeros(0, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(0, 4, device=DEV), stream=side)
    grads = layer.backward(torch.zeros_like(y), stream=side)
    with torch.cuda.stream(side):  # zeroed there, before anything that follows there
        sums = [g.abs().sum() for g in grads[2:]]
    torch.cuda.synchronize()
    assert all(float(s) == 0.0 for s in sums)


def test_status_of_a_side_stream_is_waited_for_and_reported_once():
    from paper_2609_04609_b200 import ciera

    layer, w = _layer(4, 128, 128, 2, 8)
    layer.step(w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        bad = torch.tensor([0, 64, 128, 128, 128], dtype=torch.int32, device=DEV)  # not a multiple of 128
    cap = 256
    ciera.fp8_matmul(layer.x_q[:cap], layer.x_s, layer.w1, layer.w1_s, layer.h[:cap], bad, status=layer.status, stream=side)
    with pytest.raises(ciera.CieraError) as e:
        layer.check_status()
    assert e.value.status == ciera.ERR_CORRUPT
    layer.check_status()


def test_a_refused_forward_leaves_nothing_to_go_back_through():
    from paper_2609_04609_b200 import ciera

    layer, w = _layer(4, 128, 128, 2, 8)
    layer.step(w)
    x, logits, dout = _inputs(layer, 8, 5)
    y = layer.forward(x, logits)
    with pytest.raises(ciera.CieraError):
        layer.forward(x, logits, bias=torch.zeros(3, device=DEV))
    with pytest.raises(RuntimeError):
        layer.backward(dout)
    assert torch.equal(layer.forward(x, logits), y)
    layer.backward(dout)
