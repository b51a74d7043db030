"""silu(g) * u and its gradient where 32 bits and 64 part: gates far from zero, and the gate at which the gradient vanishes."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref
from tests.test_gpu_fp8 import DEV, DTYPES, _bytes, _up

pytestmark = pytest.mark.gpu


def _rows(x, cols, kind, grad=None, layout=None):
    """Values and scale bytes of both orientations; layout: (slot_of_row, starts)"""
    from paper_2609_04609_b200 import ciera

    rows = x.shape[0]
    _, q = _bytes(rows, cols)
    _, qt = _bytes(cols, rows)
    s = torch.zeros(_up(cols, 128) // 128, rows, dtype=torch.uint8, device=DEV)
    st = torch.zeros(_up(rows, 128) // 128, cols, dtype=torch.uint8, device=DEV)
    kw = {}
    if layout:
        kw = dict(slot_of_row=layout[0].to(DEV), top_k=1, starts=layout[1].to(DEV))
    ciera.fp8_quantize_rows(x.to(DEV), q, s, qt, st, kind=kind, grad=None if grad is None else grad.to(DEV), **kw)
    torch.cuda.synchronize()
    return q, s, qt, st


def _agree(got, y, cancel=0.0):
    """Scale bytes of y (64 bits) in both orientations, values within half a step of e4m3 and 16 steps of 32 bits of the result and
    of the terms that cancel in it."""
    q, s, qt, st = got
    for q_, s_, rows in ((q, s, y), (qt, st, y.T.copy())):
        _, want = ref.quantize_rows(rows)
        assert np.array_equal(s_.cpu().numpy(), want)
        have = ref.operand_values(q_, s_).cpu().numpy()
        f = 2.0 ** (want.T.repeat(128, 1)[:, : rows.shape[1]] - 127.0)
        size = np.abs(rows) + (cancel if rows is y else np.transpose(cancel))
        off = 16 * 2.0**-24 * size
        assert (np.abs(have - rows) <= 2.0**-4 * (np.abs(rows) + off) + 2.0**-10 * f + off).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("f", [128, 130, 34])
def test_gates_far_below_zero(dtype, f):
    """silu(g) falls to e^g far beyond the smallest 32-bit number; a large u brings the product back."""
    from paper_2609_04609_b200 import ciera

    rng = np.random.default_rng(f)
    rows, dt = 130, DTYPES[dtype]
    g = rng.uniform(-190.0, -60.0, (rows, f))
    top = 4.0 if dtype == "fp16" else 37.0
    u = 10.0 ** rng.uniform(-3.0, top, (rows, f)) * rng.choice([-1.0, 1.0], (rows, f))
    g[:40] = -60.0 - 130.0 * rng.random((40, 1))  # whole rows of one gate
    g[40, :] = -87.0
    g[41, :] = -87.5
    g[42, 1:] = -300.0
    u[43, :] = 0.0
    x = torch.from_numpy(np.concatenate([g, u], 1)).to(dt)
    assert torch.isfinite(x).all()
    _agree(_rows(x, f, ciera.SOURCE_SWIGLU), ref.swiglu(x.double().numpy()))
    # gradients: the same gates, d of an ordinary size
    d = torch.from_numpy(rng.standard_normal((rows, f))).to(dt)
    if f % 2 == 0:
        y = ref.swiglu_backward(x.double().numpy(), d.double().numpy())
        _agree(_rows(x, 2 * f, ciera.SOURCE_SWIGLU_BACKWARD, d), y)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gates_far_above_zero(dtype):
    """silu(g) = g and its derivative 1, however large g is."""
    from paper_2609_04609_b200 import ciera

    rng = np.random.default_rng(4)
    rows, f = 128, 128
    g = 10.0 ** rng.uniform(1.0, 38.0, (rows, f))
    u = 10.0 ** rng.uniform(-38.0, 0.0, (rows, f))
    x = torch.from_numpy(np.concatenate([g, u], 1)).to(DTYPES[dtype])
    _agree(_rows(x, f, ciera.SOURCE_SWIGLU), ref.swiglu(x.double().numpy()))
    d = torch.from_numpy(10.0 ** rng.uniform(-3.0, 0.0, (rows, f))).to(DTYPES[dtype])
    y = ref.swiglu_backward(x.double().numpy(), d.double().numpy())
    _agree(_rows(x, 2 * f, ciera.SOURCE_SWIGLU_BACKWARD, d), y)


ROOT = -1.2784645427610738  # 1 + g (1 - sigmoid(g)) = 0


@pytest.mark.parametrize("width", [1e-4, 1e-3, 1e-2, 0.06, 0.2])
@pytest.mark.parametrize("live", ["row", "column"])
def test_gate_gradients_beside_their_root_next_to_a_border(width, live):
    """The gradient of the gate vanishes at one g: its terms cancel, and its scale is still that of 64 bits.  One value of a block is
    live, within rounding of 1.75 * 2^n, as an expert's with one token is in a transposed operand."""
    from paper_2609_04609_b200 import ciera

    rng = np.random.default_rng(int(width * 1e5))
    rows, f = 256, 128
    g = (ROOT + rng.uniform(-width, width, (rows, f))).astype(np.float32)
    g64 = g.astype(np.float64)
    s = 1 / (1 + np.exp(-g64))
    factor = s * (1 + g64 * (1 - s))
    u = (3.5 / np.abs(factor)).astype(np.float32)
    steps = rng.integers(-2, 3, (rows, f))
    for k in (1, 2):
        u = np.where(steps >= k, np.nextafter(u, np.float32(np.inf)), np.where(steps <= -k, np.nextafter(u, np.float32(0)), u))
    at = np.zeros((rows, f), bool)
    at[np.arange(rows), np.arange(rows) % f] = True  # one value in each row, and in each column of 128 rows
    u = np.where(at, u, np.float32(0.0)) if live == "column" else np.where(at, u, u * np.float32(0.3))
    x = torch.from_numpy(np.concatenate([g, u], 1))
    d = torch.ones(rows, f)
    y = ref.swiglu_backward(x.double().numpy(), d.double().numpy())
    _, want = ref.quantize_rows(y)
    assert len(np.unique(want[0])) == 2  # both sides of the border occur
    cancel = np.concatenate([np.abs(u * s), np.zeros((rows, f))], 1)
    _agree(_rows(x, 2 * f, ciera.SOURCE_SWIGLU_BACKWARD, d), y, cancel)


def test_gate_gradients_beside_their_root_in_an_experts_segment():
    """bf16 gates at the number next to the root, one token in each expert's segment."""
    from paper_2609_04609_b200 import ciera

    rows, f = 512, 256
    rng = np.random.default_rng(7)
    g = torch.full((rows, f), -1.28125, dtype=torch.bfloat16)
    g[::128, 1::2] = -1.2734375
    u = torch.from_numpy(10.0 ** rng.uniform(2.0, 5.0, (rows, f))).bfloat16()
    d = torch.from_numpy(rng.uniform(0.5, 2.0, (rows, f))).bfloat16()
    x = torch.cat([g, u], 1)
    slot = torch.full((rows,), -1, dtype=torch.int32)
    slot[::128] = torch.arange(4, dtype=torch.int32)
    starts = torch.arange(0, rows + 1, 128, dtype=torch.int32)
    y = ref.swiglu_backward(x.double().numpy(), d.double().numpy())
    y[slot < 0] = 0.0
    s = 1 / (1 + np.exp(1.28125))
    cancel = np.concatenate([np.abs((u * d).double().numpy() * s), np.zeros((rows, f))], 1)
    _agree(_rows(x, 2 * f, ciera.SOURCE_SWIGLU_BACKWARD, d, (slot, starts)), y, cancel)


@pytest.mark.parametrize("f", [128, 126, 192])
@pytest.mark.parametrize("kind", ["value", "gradient"])
def test_rows_and_columns_of_zeros_and_of_what_is_too_small(f, kind):
    """A block of zeros has byte 127, one of numbers too small for 32 bits byte 1, in both orientations."""
    from paper_2609_04609_b200 import ciera

    rng = np.random.default_rng(f)
    rows = 300
    g = rng.standard_normal((rows, f)).astype(np.float32)
    u = rng.standard_normal((rows, f)).astype(np.float32)
    d = rng.standard_normal((rows, f)).astype(np.float32)
    u[5], d[6], g[7] = 0.0, 0.0, 0.0
    g[8, ::2] = u[8, 1::2] = d[8] = 0.0
    tiny = np.float32(1e-25)
    g[9:12], u[9:12], d[9:12] = tiny, tiny, tiny  # products of 1e-50
    u[10, 1:] = d[10, 1:] = 0.0  # (one value of a row that is not a zero)
    u[128:256], d[128:256] = 0.0, 0.0  # a tile of zeros ...
    u[128:256, 3], g[128:256, 3], d[128:256, 3] = tiny, tiny, tiny  # ... but for one column ...
    u[130, 4], g[130, 4], d[130, 4] = tiny, tiny, -tiny  # ... and one value
    u[:, 7] = d[:, 7] = 0.0
    u[:128, 9], g[:128, 9], d[:128, 9] = tiny, -tiny, tiny
    u[256:], d[256:] = 0.0, 0.0
    x = torch.from_numpy(np.concatenate([g, u], 1))
    slot = torch.arange(rows, dtype=torch.int32)
    slot[[20, 140, 299]] = -1
    starts = torch.tensor([0, rows], dtype=torch.int32)
    if kind == "value":
        y = ref.swiglu(x.double().numpy())
        got = lambda layout: _rows(x, f, ciera.SOURCE_SWIGLU, None, layout)  # noqa: E731
    else:
        dd = torch.from_numpy(d)
        y = ref.swiglu_backward(x.double().numpy(), dd.double().numpy())
        got = lambda layout: _rows(x, 2 * f, ciera.SOURCE_SWIGLU_BACKWARD, dd, layout)  # noqa: E731
    assert {1, 127} <= set(np.unique(ref.quantize_rows(y)[1])) and {1, 127} <= set(np.unique(ref.quantize_rows(y.T.copy())[1]))
    _agree(got(None), y)
    y = y.copy()
    y[slot.numpy() < 0] = 0.0
    _agree(got((slot, starts)), y)
