"""Operands in e2m1 with a power of two for each 32 values of a row, bit for bit as defined."""
import numpy as np
import pytest
import torch

from tests import fp4_reference as f4
from tests import moe_reference as ref
from tests.test_gpu_fp8 import DTYPES, SENTINEL, _layout, _up

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _codes(*shape, extra=0):
    """Bytes filled with SENTINEL for [..., cols] codes, rows 16 bytes aligned, and the view of the codes."""
    line = -(-shape[-1] // 2)
    buf = torch.full((*shape[:-1], _up(line, 16) + extra), SENTINEL, dtype=torch.uint8, device=DEV)
    return buf, buf[..., :line]


def _atoms(*shape, extra=0):
    rows, cols = shape[-2:]
    buf = torch.full((*shape[:-2], -(-rows // 128), -(-cols // 128) + extra, 512), SENTINEL, dtype=torch.uint8, device=DEV)
    return buf, buf[..., : -(-cols // 128), :]


def _check(buf, q, atoms_buf, atoms, want, rows_there=None):
    """Codes and scale bytes as in `want` (float64 [rows, cols]), 127 behind a row's last group, all else left as it was."""
    rows, cols = want.shape
    there = np.arange(rows) if rows_there is None else rows_there
    codes, s = f4.quantize(want[there])
    have = f4.unpack(q, cols)[there]
    assert np.array_equal(f4.scale_bytes(atoms, rows, cols)[there], s)
    nan = np.repeat(s == 255, 32, 1)[:, :cols]
    assert np.array_equal(np.where(nan, 0, codes), have)
    if cols % 2:
        assert (q[:, -1].cpu().numpy()[there] >> 4 == 0).all()
    assert (buf[:, q.shape[1] :] == SENTINEL).all()
    left = np.ones(rows, bool)
    left[there] = False
    assert (q.cpu().numpy()[left] == SENTINEL).all()
    full = np.full((atoms.shape[0], atoms.shape[1], 512), SENTINEL, np.uint8)
    exact = f4.to_atoms(s)
    for i, r in enumerate(there):
        at = 16 * (r % 32) + 4 * (r % 128 // 32)
        src = 16 * (i % 32) + 4 * (i % 128 // 32)
        full[r // 128, :, at : at + 4] = exact[i // 128, :, src : src + 4]
    assert np.array_equal(atoms.cpu().numpy(), full)
    assert (atoms_buf[:, atoms.shape[1] :] == SENTINEL).all()


def _values(rows, cols, dtype, seed):
    """Values over many magnitudes: ordinary rows, tiny and huge ones, zeros, largest values next to a power's border."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    dt = DTYPES[dtype]
    if rows > 9:
        top = float(torch.finfo(dt).max)
        x[1] = 0.0
        x[2] *= 2.0**-20 if dtype == "fp16" else 2.0**-130
        x[3] = x[3] / x[3].abs().max() * top * 0.99
        x[4, 0], x[4, 1:] = 3.0, x[4, 1:] * 0.1  # 6 * 2^-1: on the border
        x[5, 0], x[5, 1:] = 3.0 + 3.0 * torch.finfo(dt).eps * 2, x[5, 1:] * 0.1  # just above
        x[6] *= 1e-3
        x[6, -1] = 500.0
        x[7] = 0.0
        x[7, cols // 2] = float(torch.finfo(dt).smallest_normal) / 2  # subnormal
        x[8, ::2], x[8, 1::2] = -0.25, 0.75  # ties
        x[9, cols // 3] = float("nan") if cols % 2 else float("inf")
    return x.to(dt)


@pytest.mark.parametrize("rows,cols,dtype,strided", [
    (1, 1, "bf16", False), (1, 128, "fp32", False), (130, 256, "bf16", False), (100, 300, "fp16", True), (257, 77, "fp32", False),
    (64, 129, "bf16", True), (128, 2048, "bf16", False), (33, 131, "fp16", False), (300, 515, "bf16", True), (40, 1000, "fp32", True),
    (31, 34, "fp16", False), (2, 33, "fp32", False),
])
def test_rows_equal_the_definition(rows, cols, dtype, strided):
    from paper_2609_04609_b200 import ciera

    x = _values(rows, cols, dtype, rows + cols)
    dev = x.to(DEV)
    if strided:
        dev = torch.cat([dev, dev[:, :3]], 1)[:, :cols]
    buf, q = _codes(rows, cols, extra=16)
    atoms_buf, atoms = _atoms(rows, cols, extra=1)
    ciera.fp4_quantize_rows(dev, q, atoms)
    torch.cuda.synchronize()
    _check(buf, q, atoms_buf, atoms, x.double().numpy())


def test_every_bf16_pattern_is_rounded_as_defined():
    """Each pattern as the largest of a group of its own and below a fixed largest value."""
    from paper_2609_04609_b200 import ciera

    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    for top in (None, 1.0, 6.0, 2.0**-100):
        x = torch.zeros(65536, 2, dtype=torch.bfloat16)
        x[:, 0] = bits
        if top is not None:
            x[:, 1] = top
        buf, q = _codes(65536, 2)
        _, atoms = _atoms(65536, 2)
        ciera.fp4_quantize_rows(x.to(DEV), q, atoms)
        codes, s = f4.quantize(x.double().numpy())
        assert np.array_equal(f4.scale_bytes(atoms, 65536, 2), s)
        assert np.array_equal(np.where(s == 255, 0, codes), f4.unpack(q, 2))


@pytest.mark.parametrize("source", ["gather", "swiglu"])
@pytest.mark.parametrize("T,k,E,cols,dtype", [(1, 2, 4, 256, "bf16"), (77, 3, 5, 130, "bf16"), (200, 8, 16, 384, "fp32"), (50, 2, 3, 33, "fp16")])
def test_rows_of_a_layout(source, T, k, E, cols, dtype):
    from paper_2609_04609_b200 import ciera

    dt = DTYPES[dtype]
    starts, slot, cap = _layout(T, k, E, T)
    used = int(starts[-1])
    g = torch.Generator().manual_seed(cols)
    buf, q = _codes(cap, cols)
    atoms_buf, atoms = _atoms(cap, cols)
    there = (slot[:used] >= 0).numpy()
    want = np.zeros((cap, cols))
    if source == "gather":
        x = torch.randn(T, cols, generator=g).to(dt)
        want[:used][there] = x.double().numpy()[slot[:used][there].numpy() // k]
    else:
        x = torch.randn(cap, 2 * cols, generator=g).to(dt)
        x[5 % cap, :cols] = -100.0  # silu's exponential leaves 32 bits
        x[6 % cap] = 0.0
        want[:used][there] = ref.swiglu(x.double().numpy()[:used][there])
    ciera.fp4_quantize_rows(x.to(DEV), q, atoms, kind=ciera.SOURCE_SWIGLU if source == "swiglu" else ciera.SOURCE_ROWS,
                            slot_of_row=slot.to(DEV), top_k=k, starts=starts.to(DEV))
    torch.cuda.synchronize()
    if source == "gather":
        _check(buf, q, atoms_buf, atoms, want, np.arange(used))
        return
    # scales are those of 64 bits; values are off by at most 20 steps of 32 bits before the rounding, half a step of which is at
    # most 2^-2 of the value (a bit behind the point) or 2^-2 of the scale
    _, s = f4.quantize(want[:used])
    assert np.array_equal(f4.scale_bytes(atoms, cap, cols)[:used], s)
    unit = np.repeat(2.0 ** (s - 127.0), 32, 1)[:, :cols]
    have = f4.values(f4.unpack(q, cols)[:used], s)
    assert (np.abs(have - want[:used]) <= np.maximum(np.abs(want[:used]) / 4, unit / 4) * (1 + 2.0**-18)).all()
    assert (q[used:] == SENTINEL).all() and (atoms[used // 128 :] == SENTINEL).all()


def test_groups_next_to_a_border_of_silu():
    """The largest value a step of 64 bits above or below 6 * 2^s: gates and ups that bring silu(g) * u there."""
    from paper_2609_04609_b200 import ciera

    rows = 256
    gate = torch.linspace(-8.0, 8.0, rows, dtype=torch.float64).float()
    gate[gate.abs() < 1e-3] = 0.5
    silu = gate.double() / (1 + torch.exp(-gate.double()))
    up = (3.0 / silu).float()
    up = torch.where(torch.arange(rows) % 3 == 0, torch.nextafter(up, torch.zeros(())), up)
    up = torch.where(torch.arange(rows) % 3 == 1, torch.nextafter(up, up * 2), up)
    x = torch.zeros(rows, 64)
    x[:, 3], x[:, 32 + 3] = gate, up
    _, q = _codes(rows, 32)
    _, atoms = _atoms(rows, 32)
    ciera.fp4_quantize_rows(x.to(DEV), q, atoms, kind=ciera.SOURCE_SWIGLU)
    _, s = f4.quantize(ref.swiglu(x.double().numpy()))
    assert len(np.unique(s)) == 2  # both sides are there
    assert np.array_equal(f4.scale_bytes(atoms, rows, 32), s)


@pytest.mark.parametrize("m,rows,cols,dtype,strided", [
    (1, 1, 1, "bf16", False), (2, 128, 128, "bf16", False), (3, 100, 70, "bf16", True), (2, 130, 257, "fp16", False),
    (1, 64, 200, "fp32", False), (2, 33, 65, "fp32", True), (1, 300, 128, "fp16", True), (5, 256, 384, "bf16", False),
])
def test_matrices_both_ways(m, rows, cols, dtype, strided):
    from paper_2609_04609_b200 import ciera

    x = torch.stack([_values(rows, cols, dtype, 7 * i + rows) for i in range(m)])
    dev = x.to(DEV)
    if strided:
        dev = torch.cat([dev, dev], 2)[:, :, :cols]
    for both in (True, False):
        buf, q = _codes(m, rows, cols, extra=16)
        abuf, atoms = _atoms(m, rows, cols, extra=1)
        tbuf, qt = _codes(m, cols, rows, extra=16)
        tabuf, atoms_t = _atoms(m, cols, rows, extra=1)
        if both:
            ciera.fp4_quantize_matrices(dev, q, atoms, qt, atoms_t)
        else:
            ciera.fp4_quantize_matrices(dev, qt=qt, scales_t=atoms_t)
        torch.cuda.synchronize()
        for i in range(m):
            if both:
                _check(buf[i], q[i], abuf[i], atoms[i], x[i].double().numpy())
            _check(tbuf[i], qt[i], tabuf[i], atoms_t[i], x[i].double().numpy().T.copy())
        if not both:
            assert (buf == SENTINEL).all() and (abuf == SENTINEL).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols,strided", [(1, 1, False), (130, 300, False), (257, 77, True), (64, 256, True), (1, 4096, False)])
def test_values_of_every_code_and_scale(rows, cols, strided, dtype):
    from paper_2609_04609_b200 import ciera

    g = np.random.default_rng(rows)
    codes = g.integers(0, 16, (rows, cols))
    s = g.integers(100, 140, (rows, -(-cols // 32)))
    s.reshape(-1)[: min(256, s.size)] = np.arange(min(256, s.size))[::-1]  # all bytes, NaN and the subnormal one among them
    q, atoms = f4.operand_tensors(codes, s, DEV)
    out = torch.full((rows, cols + (3 if strided else 0)), 7.0, dtype=DTYPES[dtype], device=DEV)
    view = out[:, :cols]
    ciera.fp4_values(q, atoms, view)
    want = torch.from_numpy(f4.values(codes, s)).to(DTYPES[dtype])
    assert torch.equal(torch.nan_to_num(view.cpu(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
    assert (out[:, cols:] == 7.0).all()


def test_values_of_a_stack():
    from paper_2609_04609_b200 import ciera

    x = torch.randn(3, 200, 96, device=DEV)
    buf, q = _codes(3, 200, 96)
    _, atoms = _atoms(3, 200, 96)
    ciera.fp4_quantize_matrices(x, q, atoms)
    out = torch.zeros(3, 200, 96, device=DEV)
    ciera.fp4_values(q, atoms, out)
    for i in range(3):
        codes, s = f4.quantize(x[i].double().cpu().numpy())
        assert np.array_equal(out[i].double().cpu().numpy(), f4.values(codes, s))
