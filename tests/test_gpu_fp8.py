"""Operands in e4m3 with a power of two for each block of 128 values, and their products."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E4M3 = torch.float8_e4m3fn
SENTINEL = 0x55


def _up(a, b):
    return -(-a // b) * b


def _bytes(rows, cols, extra=0):
    """A byte tensor filled with SENTINEL, rows 16 bytes aligned, and the view [rows, cols] as e4m3."""
    buf = torch.full((rows, _up(cols, 16) + extra), SENTINEL, dtype=torch.uint8, device=DEV)
    return buf, buf[:, :cols].view(E4M3)


def _values(q):
    return ref.e4m3_values()[q.view(torch.uint8).cpu().numpy()]


def _same(got, want):
    return np.array_equal(got, want, equal_nan=True)


def _rows_case(rows, cols, dtype, seed):
    """Values over many magnitudes: ordinary rows, tiny and huge ones, zeros, largest values next to a power's border."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64)
    dt = DTYPES[dtype]
    if rows > 8:
        top = float(torch.finfo(dt).max)
        x[1] = 0.0
        x[2] *= 2.0**-20 if dtype == "fp16" else 2.0**-130
        x[3] = x[3] / x[3].abs().max() * top * 0.99
        x[4, 0] = 3.5  # 448 * 2^-7: on the border
        x[4, 1:] *= 0.1
        x[5, 0] = 3.5 + 3.5 * torch.finfo(dt).eps * 2  # just above
        x[5, 1:] *= 0.1
        x[6] *= 1e-3
        x[6, -1] = 500.0
        x[7] = 0.0
        x[7, cols // 2] = float(torch.finfo(dt).smallest_normal) / 2  # subnormal
    return x.to(dt)


@pytest.mark.parametrize("rows,cols,dtype,turned,strided", [
    (1, 1, "bf16", True, False), (1, 128, "fp32", False, False), (130, 256, "bf16", True, False), (100, 300, "fp16", True, True),
    (257, 77, "fp32", True, False), (64, 129, "bf16", False, True), (128, 2048, "bf16", True, False), (33, 131, "fp16", False, False),
    (300, 515, "bf16", True, True),
])
def test_rows_equal_the_definition(rows, cols, dtype, turned, strided):
    from paper_2609_04609_b200 import ciera

    x = _rows_case(rows, cols, dtype, rows + cols)
    dev = x.to(DEV)
    if strided:
        dev = torch.cat([dev, dev[:, :3]], 1)[:, :cols]
    qb, q = _bytes(rows, cols, 16)
    sb = torch.full((_up(cols, 128) // 128, rows + 5), SENTINEL, dtype=torch.uint8, device=DEV)
    qtb, qt = _bytes(cols, rows, 16)
    stb = torch.full((_up(rows, 128) // 128, cols + 5), SENTINEL, dtype=torch.uint8, device=DEV)
    ciera.fp8_quantize_rows(dev, q, sb, qt if turned else None, stb if turned else None)
    torch.cuda.synchronize()
    want, s = ref.quantize_rows(x.double().numpy())
    assert np.array_equal(sb[:, :rows].cpu().numpy(), s) and _same(_values(q), want)
    assert (qb[:, cols:] == SENTINEL).all() and (sb[:, rows:] == SENTINEL).all()
    if turned:
        want, s = ref.quantize_rows(x.double().numpy().T.copy())
        assert np.array_equal(stb[:, :cols].cpu().numpy(), s) and _same(_values(qt), want)
        assert (qtb[:, rows:] == SENTINEL).all() and (stb[:, cols:] == SENTINEL).all()


def test_every_bf16_pattern_is_rounded_as_defined():
    """Each pattern as the largest of a block of its own and below a fixed largest value."""
    from paper_2609_04609_b200 import ciera

    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    for top in (None, 1.0, 448.0, 2.0**-100):
        x = torch.zeros(65536, 2, dtype=torch.bfloat16)
        x[:, 0] = bits
        if top is not None:
            x[:, 1] = top
        _, q = _bytes(65536, 2)
        s = torch.zeros(1, 65536, dtype=torch.uint8, device=DEV)
        ciera.fp8_quantize_rows(x.to(DEV), q, s)
        want, ws = ref.quantize_rows(x.double().numpy())
        assert np.array_equal(s.cpu().numpy(), ws)
        assert _same(_values(q), want)


def _layout(T, k, E, seed, dropped=0.1):
    g = torch.Generator().manual_seed(seed)
    ids = torch.rand(T, E, generator=g).topk(k, 1).indices.int()
    ids = torch.where(torch.rand(T, k, generator=g) < dropped, torch.full_like(ids, -1), ids)
    starts, counts, ros, sor = ref.layout(ids, E)
    cap = starts[-1] + 200
    slot = torch.full((cap,), 12345678, dtype=torch.int32)  # behind the last segment: never followed
    for r, v in sor.items():
        slot[r] = v
    return torch.tensor(starts, dtype=torch.int32), slot, cap


@pytest.mark.parametrize("source", ["gather", "weighted", "swiglu", "swiglu_backward"])
@pytest.mark.parametrize("T,k,E,cols,dtype", [(1, 2, 4, 256, "bf16"), (77, 3, 5, 130, "bf16"), (200, 8, 16, 384, "fp32"), (50, 2, 3, 34, "fp16")])
def test_rows_of_a_layout(source, T, k, E, cols, dtype):
    from paper_2609_04609_b200 import ciera

    dt = DTYPES[dtype]
    starts, slot, cap = _layout(T, k, E, T)
    used = int(starts[-1])
    g = torch.Generator().manual_seed(cols)
    kw, weights, grad = {}, None, None
    live = [r for r in range(used) if slot[r] >= 0]
    y = np.zeros((used, cols))
    at = slot[live].long()
    if source in ("gather", "weighted"):
        x = torch.randn(T, cols, generator=g).to(dt)
        y[live] = x.double().numpy()[at // k]
        kw["kind"] = ciera.SOURCE_ROWS
        if source == "weighted":
            weights = torch.rand(T, k, generator=g)
            # the product is rounded to 32 bits before anything else is done with it
            y[live] = (x.float()[at // k] * weights.reshape(-1)[at][:, None]).double().numpy()
    else:
        f = cols if source == "swiglu" else cols // 2
        x = (torch.randn(cap, 2 * f, generator=g) * 2).to(dt)
        kw["kind"] = ciera.SOURCE_SWIGLU
        x64 = x.double().numpy()
        if source == "swiglu":
            y[live] = ref.swiglu(x64)[live]
        else:
            grad = torch.randn(cap, f, generator=g).to(dt)
            kw["kind"] = ciera.SOURCE_SWIGLU_BACKWARD
            y[live] = ref.swiglu_backward(x64, grad.double().numpy())[live]
        x[[r for r in range(cap) if r not in set(live)]] = float("nan")  # rows without a slot are not read
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    qb, q = _bytes(cap, cols)
    qtb, qt = _bytes(cols, cap)
    sb = torch.full((_up(cols, 128) // 128, cap), SENTINEL, dtype=torch.uint8, device=DEV)
    stb = torch.full((_up(cap, 128) // 128, cols), SENTINEL, dtype=torch.uint8, device=DEV)
    ciera.fp8_quantize_rows(dev(x), q, sb, qt, stb, grad=dev(grad), slot_of_row=dev(slot), top_k=k, row_weights=dev(weights),
                            starts=dev(starts), **kw)
    torch.cuda.synchronize()
    for got, scales, rows64, lines in ((q[:used], sb[:, :used], y, used), (qt[:, :used], stb[: used // 128], y.T.copy(), cols)):
        want, s = ref.quantize_rows(rows64)
        assert np.array_equal(scales[:, :lines].cpu().numpy(), s)
        if "swiglu" not in source:
            assert _same(_values(got), want)
        else:
            # 32 bits before the rounding: half a step of e4m3, 20 steps of 32 bits of the terms (at most 16 times the result's
            # size before they cancel); below the least exponent the step is fixed
            have = ref.operand_values(got, scales).cpu().numpy()
            f = 2.0 ** (s.T.repeat(128, 1)[:, : rows64.shape[1]] - 127.0)
            size = np.abs(rows64) + (16 * 20 * 2.0**-24 * np.abs(rows64).max() if source == "swiglu_backward" else 0)
            assert (np.abs(have - rows64) <= np.maximum(2.0**-4 * size, 2.0**-10 * f) * 1.001 + 16 * 20 * 2.0**-24 * size).all()
    # rows behind the last segment are left as they were
    assert (qb[used:] == SENTINEL).all() and (sb[:, used:] == SENTINEL).all()
    assert (qtb[:, used:] == SENTINEL).all() and (stb[used // 128 :] == SENTINEL).all()


def test_swiglu_scales_next_to_a_border():
    """Largest values within 32-bit rounding of 1.75 * 2^n: the scale is that of 64 bits, in both orientations."""
    from paper_2609_04609_b200 import ciera

    rng = np.random.default_rng(0)
    rows, f = 256, 128
    g = rng.uniform(0.5, 3.0, (rows, f)).astype(np.float32)
    target = np.float64(3.5)
    u = (target / (g.astype(np.float64) / (1 + np.exp(-g.astype(np.float64))))).astype(np.float32)
    u[:, 1:] *= np.float32(0.01)
    u[::2, 0] = np.nextafter(u[::2, 0], np.float32(9))
    x = torch.from_numpy(np.concatenate([g, u], 1))
    _, q = _bytes(rows, f)
    s = torch.zeros(1, rows, dtype=torch.uint8, device=DEV)
    _, qt = _bytes(f, rows)
    st = torch.zeros(2, f, dtype=torch.uint8, device=DEV)
    ciera.fp8_quantize_rows(x.to(DEV), q, s, qt, st, kind=ciera.SOURCE_SWIGLU)
    y = ref.swiglu(x.double().numpy())
    assert np.array_equal(s.cpu().numpy(), ref.quantize_rows(y)[1])
    assert len(np.unique(s.cpu().numpy())) == 2  # both sides of the border occur
    assert np.array_equal(st.cpu().numpy(), ref.quantize_rows(y.T.copy())[1])


@pytest.mark.parametrize("m,rows,cols,dtype,turned", [
    (1, 1, 1, "fp32", True), (3, 128, 128, "bf16", True), (2, 300, 200, "bf16", True), (2, 200, 77, "fp16", False), (5, 64, 515, "fp32", True),
])
def test_blocks_equal_the_definition(m, rows, cols, dtype, turned):
    from paper_2609_04609_b200 import ciera

    g = torch.Generator().manual_seed(rows)
    x = (torch.randn(m, rows, cols, generator=g) * 0.02).to(DTYPES[dtype])
    if cols > 200:
        x[0, :128, 128:256] = 0
        x[1, 3, 2] = float("inf")
        x[1, 40, 200] = float("nan")
    # matrices of a larger allocation: strides of rows and matrices of their own
    big = torch.zeros(m, rows + 2, cols + 7, dtype=x.dtype, device=DEV)
    big[:, :rows, :cols] = x.to(DEV)
    qb = torch.full((m, rows + 1, _up(cols, 16) + 16), SENTINEL, dtype=torch.uint8, device=DEV)
    qtb = torch.full((m, cols + 1, _up(rows, 16) + 16), SENTINEL, dtype=torch.uint8, device=DEV)
    rb, cb = _up(rows, 128) // 128, _up(cols, 128) // 128
    s = torch.full((m, rb, cb), SENTINEL, dtype=torch.uint8, device=DEV)
    st = torch.full((m, cb, rb), SENTINEL, dtype=torch.uint8, device=DEV)
    q, qt = qb[:, :rows, :cols].view(E4M3), qtb[:, :cols, :rows].view(E4M3)
    ciera.fp8_quantize_blocks(big[:, :rows, :cols], q, s, qt if turned else None, st if turned else None)
    torch.cuda.synchronize()
    for i in range(m):
        want, ws = ref.quantize_blocks(x[i].double().numpy())
        assert np.array_equal(s[i].cpu().numpy(), ws) and _same(_values(q[i]), want)
        if turned:
            assert np.array_equal(st[i].cpu().numpy(), ws.T) and _same(_values(qt[i]), want.T)
    assert (qb[:, rows:] == SENTINEL).all() and (qb[:, :, cols:] == SENTINEL).all()
    if turned:
        assert (qtb[:, cols:] == SENTINEL).all() and (qtb[:, :, rows:] == SENTINEL).all()


# ------------------------------------------------------------------------------------------------ products


def _operand(rows, cols, seed, std=1.0, pad=0):
    """Random e4m3 rows with random scale bytes around 127, on the device."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.full((rows, _up(cols, 16) + pad), 0x7F, dtype=torch.uint8, device=DEV)  # NaN behind the rows' ends: never read
    q = (torch.randn(rows, cols, generator=g, device=DEV) * 60 * std).clamp(-448, 448).to(E4M3)
    buf[:, :cols] = q.view(torch.uint8)
    nb = _up(cols, 128) // 128
    s = torch.full((nb, _up(rows, 16)), 255, dtype=torch.uint8, device=DEV)
    s[:, :rows] = torch.randint(118, 128, (nb, rows), generator=g, device=DEV, dtype=torch.uint8)
    return buf[:, :cols].view(E4M3), s


def _matrices(m, n, k, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.full((m, n, _up(k, 16)), 0x7F, dtype=torch.uint8, device=DEV)
    buf[:, :, :k] = (torch.randn(m, n, k, generator=g, device=DEV) * 60).clamp(-448, 448).to(E4M3).view(torch.uint8)
    s = torch.randint(118, 128, (m, _up(n, 128) // 128, _up(k, 128) // 128), generator=g, device=DEV, dtype=torch.uint8)
    return buf[:, :, :k].view(E4M3), s


def _close(out, a, b):
    """a [m, k], b [n, k] float64: k products (exact in 32 bits) and k additions in 32 bits in any order, then one rounding."""
    want = a @ b.t()
    size = a.abs() @ b.abs().t()
    k = a.shape[1]
    step = torch.finfo(out.dtype).eps / 2
    tol = (k + 2) * 2.0**-24 * size + step * want.abs() + (1e-7 if out.dtype == torch.float16 else 0)
    return bool(((out.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("b_rows", [False, True])
@pytest.mark.parametrize("m,n,k,out", [
    (1, 1, 1, "fp32"), (1, 128, 128, "bf16"), (1, 2048, 2048, "bf16"), (128, 256, 128, "fp32"), (129, 257, 129, "bf16"), (300, 200, 500, "fp32"),
    (1000, 77, 2049, "bf16"), (64, 640, 1111, "fp16"), (513, 1025, 640, "fp32"), (127, 383, 4096, "fp32"),
])
def test_dense_product(b_rows, m, n, k, out):
    from paper_2609_04609_b200 import ciera

    a, sa = _operand(m, k, m + k, pad=16)
    if b_rows:
        b, sb = _operand(n, k, n + k + 1)
        vb = ref.operand_values(b, sb)
    else:
        b, sb = _matrices(1, n, k, n + k + 1)
        vb = ref.matrix_values(b, sb)[0]
    o = torch.full((m + 1, n + 3), 9.0, dtype=DTYPES[out], device=DEV)
    if out == "fp16":  # within the type's range
        sa[:, :m] -= 10
    ciera.fp8_matmul(a, sa, b, sb, o[:m, :n])
    torch.cuda.synchronize()
    assert (o[m] == 9.0).all() and (o[:, n:] == 9.0).all()
    assert _close(o[:m, :n], ref.operand_values(a, sa), vb)


SEGMENTS = [[128], [0, 128, 0], [256, 0, 384, 128, 0], [128] * 9 + [0] * 7 + [640], [0, 0, 0], [1280, 0, 128]]


@pytest.mark.parametrize("segments", SEGMENTS, ids=lambda s: "-".join(map(str, s))[:24])
@pytest.mark.parametrize("n,k,out", [(128, 128, "bf16"), (300, 200, "fp32"), (2048, 384, "bf16"), (77, 1030, "fp32")])
def test_product_by_segments_of_rows(segments, n, k, out):
    from paper_2609_04609_b200 import ciera

    E = len(segments)
    starts = torch.tensor([0] + list(np.cumsum(segments)), dtype=torch.int32, device=DEV)
    used = int(starts[-1])
    rows = used + 130
    a, sa = _operand(rows, k, k)
    a.view(torch.uint8)[used:] = 0x7F
    b, sb = _matrices(E, n, k, n)
    o = torch.full((rows, n), 9.0, dtype=DTYPES[out], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ciera.fp8_matmul(a, sa, b, sb, o, starts, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    va, vb = ref.operand_values(a, sa), ref.matrix_values(b, sb)
    for e in range(E):
        lo, hi = int(starts[e]), int(starts[e + 1])
        if hi > lo:
            assert _close(o[lo:hi], va[lo:hi], vb[e]), f"expert {e}"
    assert (o[used:] == 9.0).all()  # rows behind the last segment are left as they were


@pytest.mark.parametrize("segments", SEGMENTS, ids=lambda s: "-".join(map(str, s))[:24])
@pytest.mark.parametrize("m,n,out", [(128, 128, "bf16"), (300, 200, "fp32"), (77, 1030, "fp32"), (1, 5, "bf16")])
def test_product_by_segments_of_the_contraction(segments, m, n, out):
    from paper_2609_04609_b200 import ciera

    E = len(segments)
    starts = torch.tensor([0] + list(np.cumsum(segments)), dtype=torch.int32, device=DEV)
    used = int(starts[-1])
    rows = used + 130
    a, sa = _operand(m, rows, m)
    b, sb = _operand(n, rows, n + 7)
    a.view(torch.uint8)[:, used:] = 0x7F
    o = torch.full((E, m, n), 9.0, dtype=DTYPES[out], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ciera.fp8_matmul(a, sa, b, sb, o, starts, contract=True, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    va, vb = ref.operand_values(a, sa), ref.operand_values(b, sb)
    for e in range(E):
        lo, hi = int(starts[e]), int(starts[e + 1])
        if hi == lo:
            assert (o[e] == 0).all()
        else:
            assert _close(o[e], va[:, lo:hi], vb[:, lo:hi]), f"expert {e}"


def test_product_carries_infinite_blocks_as_nan():
    from paper_2609_04609_b200 import ciera

    x = torch.randn(130, 300, device=DEV)
    x[7, 200] = float("inf")
    x[129, 5] = float("nan")
    q = torch.zeros(130, 304, dtype=torch.uint8, device=DEV)[:, :300].view(E4M3)
    s = torch.zeros(3, 144, dtype=torch.uint8, device=DEV)
    ciera.fp8_quantize_rows(x, q, s)
    b, sb = _matrices(1, 200, 300, 1)
    o = torch.zeros(130, 200, device=DEV)
    ciera.fp8_matmul(q, s, b, sb, o)
    bad = torch.isnan(o)
    assert bad[7].all() and bad[129].all() and int(bad.sum()) == 400


@pytest.mark.parametrize("contract", [False, True])
def test_bad_starts_are_reported_and_nothing_is_written(contract):
    from paper_2609_04609_b200 import ciera

    rows, k, n = 512, 128, 128
    a, sa = _operand(k, rows, 1) if contract else _operand(rows, k, 1)
    b, sb = _operand(n, rows, 2) if contract else _matrices(3, n, k, 2)
    o = torch.full((3, k, n) if contract else (rows, n), 9.0, device=DEV)
    for bad in ([0, 100, 256, 384], [128, 256, 384, 512], [0, 256, 128, 384], [0, 128, 256, 640], [0, -128, 0, 128],
                [0, 128, 256, 2**31 - 128]):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        ciera.fp8_matmul(a, sa, b, sb, o, torch.tensor(bad, dtype=torch.int32, device=DEV), contract=contract, status=status)
        torch.cuda.synchronize()
        assert status.item() == ciera.ERR_CORRUPT and (o == 9.0).all()


def test_products_from_a_graph_and_on_two_streams():
    from paper_2609_04609_b200 import ciera

    rows, n, k, E = 1024, 256, 256, 4
    a, sa = _operand(rows, k, 3)
    b, sb = _matrices(E, n, k, 4)
    starts = torch.tensor([0, 256, 256, 640, 1024], dtype=torch.int32, device=DEV)
    o = torch.zeros(rows, n, device=DEV)
    ciera.fp8_matmul(a, sa, b, sb, o, starts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ciera.fp8_matmul(a, sa, b, sb, o, starts)
    va, vb = ref.operand_values(a, sa), ref.matrix_values(b, sb)
    for cut in ([0, 0, 0, 0, 128], [0, 128, 256, 384, 512], [0, 1024, 1024, 1024, 1024]):
        starts.copy_(torch.tensor(cut, dtype=torch.int32))
        o.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        for e in range(E):
            assert cut[e] == cut[e + 1] or _close(o[cut[e] : cut[e + 1]], va[cut[e] : cut[e + 1]], vb[e])
        assert (o[cut[-1] :] == 9.0).all()
    # two calls at once
    starts.copy_(torch.tensor([0, 256, 256, 640, 1024], dtype=torch.int32))
    torch.cuda.synchronize()
    outs, streams = [torch.zeros(rows, n, device=DEV) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, out in zip(streams, outs):
            ciera.fp8_matmul(a, sa, b, sb, out, starts, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    for e, (lo, hi) in enumerate(((0, 256), (256, 256), (256, 640), (640, 1024))):
        assert lo == hi or _close(outs[0][lo:hi], va[lo:hi], vb[e])
