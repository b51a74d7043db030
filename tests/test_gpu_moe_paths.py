"""Sizes at which the kernels of the MoE layer go round their loops, and forms of operands that other tests do not reach."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref
from tests.test_gpu_fp8 import DEV, DTYPES, E4M3, SENTINEL, _bytes, _layout, _same, _up, _values
from tests.test_gpu_route import _config, _logits

pytestmark = pytest.mark.gpu


def _check_rows(q, s, y, used):
    want, ws = ref.quantize_rows(y)
    assert np.array_equal(s[:, :used].cpu().numpy(), ws) and _same(_values(q), want)


@pytest.mark.parametrize("rows,cols,dtype,turned", [
    (1500, 2056, "bf16", True), (2000, 1160, "fp16", False), (40000, 8, "bf16", False), (129, 20480, "bf16", True), (20001, 128, "fp16", True),
])
def test_rows_of_several_tiles_a_block(rows, cols, dtype, turned):
    """More tiles than the GPU has SMs, in rows of tiles that end inside a block's share."""
    from paper_2609_04609_b200 import ciera

    g = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, cols, generator=g)
    x *= torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g).float())
    x[::7, ::11] = 0
    x = x.to(DTYPES[dtype])
    qb, q = _bytes(rows, cols, 16)
    sb = torch.full((_up(cols, 128) // 128, rows + 5), SENTINEL, dtype=torch.uint8, device=DEV)
    qtb, qt = _bytes(cols, rows, 16)
    stb = torch.full((_up(rows, 128) // 128, cols + 5), SENTINEL, dtype=torch.uint8, device=DEV)
    ciera.fp8_quantize_rows(x.to(DEV), q, sb, qt if turned else None, stb if turned else None)
    torch.cuda.synchronize()
    _check_rows(q, sb, x.double().numpy(), rows)
    assert (qb[:, cols:] == SENTINEL).all() and (sb[:, rows:] == SENTINEL).all()
    if turned:
        _check_rows(qt, stb, x.double().numpy().T.copy(), cols)
        assert (qtb[:, rows:] == SENTINEL).all() and (stb[:, cols:] == SENTINEL).all()
    else:
        assert (qtb == SENTINEL).all() and (stb == SENTINEL).all()


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_gathered_rows_of_several_tiles_a_block(dtype, weighted):
    from paper_2609_04609_b200 import ciera

    T, k, E, cols = 900, 4, 20, 1032
    starts, slot, cap = _layout(T, k, E, 5)
    used = int(starts[-1])
    g = torch.Generator().manual_seed(6)
    x = torch.randn(T, cols, generator=g).to(DTYPES[dtype])
    w = torch.rand(T, k, generator=g) if weighted else None
    live = np.array([r for r in range(used) if slot[r] >= 0])
    at = slot[live].long()
    y = np.zeros((used, cols))
    y[live] = (x.float()[at // k] * w.reshape(-1)[at][:, None] if weighted else x.float()[at // k]).double().numpy()
    qb, q = _bytes(cap, cols)
    qtb, qt = _bytes(cols, cap)
    sb = torch.full((_up(cols, 128) // 128, cap), SENTINEL, dtype=torch.uint8, device=DEV)
    stb = torch.full((_up(cap, 128) // 128, cols), SENTINEL, dtype=torch.uint8, device=DEV)
    ciera.fp8_quantize_rows(x.to(DEV), q, sb, qt, stb, slot_of_row=slot.to(DEV), top_k=k, starts=starts.to(DEV),
                            row_weights=None if w is None else w.to(DEV))
    torch.cuda.synchronize()
    _check_rows(q[:used], sb, y, used)
    want, ws = ref.quantize_rows(y.T.copy())
    assert np.array_equal(stb[: used // 128].cpu().numpy(), ws) and _same(_values(qt[:, :used]), want)
    assert (qb[used:] == SENTINEL).all() and (sb[:, used:] == SENTINEL).all()
    assert (qtb[:, used:] == SENTINEL).all() and (stb[used // 128 :] == SENTINEL).all()


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m,rows,cols", [(1, 128, 128), (3, 300, 212), (2, 4, 4), (5, 132, 516), (1, 127, 1024)])
def test_aligned_blocks_equal_the_definition(m, rows, cols, dtype, turned):
    """Rows that start at multiples of four values, edges inside the last blocks, matrices of a larger allocation."""
    from paper_2609_04609_b200 import ciera

    g = torch.Generator().manual_seed(rows + cols)
    x = (torch.randn(m, rows, cols, generator=g) * 0.02).to(DTYPES[dtype])
    x[0, 3, 2] = -2.0
    if m > 2:
        x[0, :128, 128:256] = 0
        x[1, 3, 2] = float("-inf")
        x[1, 131, 200] = float("nan")
        x[2, 130, 130] = torch.finfo(x.dtype).max
    big = torch.full((m, rows + 2, cols + 8), float("nan"), dtype=x.dtype, device=DEV)
    big[:, :rows, :cols] = x.to(DEV)
    qb = torch.full((m, rows + 1, _up(cols, 16) + 16), SENTINEL, dtype=torch.uint8, device=DEV)
    qtb = torch.full((m, cols + 1, _up(rows, 16) + 16), SENTINEL, dtype=torch.uint8, device=DEV)
    rb, cb = _up(rows, 128) // 128, _up(cols, 128) // 128
    s = torch.full((m, rb, cb + 1), SENTINEL, dtype=torch.uint8, device=DEV)
    st = torch.full((m, cb, rb + 1), SENTINEL, dtype=torch.uint8, device=DEV)
    q, qt = qb[:, :rows, :cols].view(E4M3), qtb[:, :cols, :rows].view(E4M3)
    ciera.fp8_quantize_blocks(big[:, :rows, :cols], q, s[:, :, :cb], qt if turned else None, st[:, :, :rb] if turned else None)
    torch.cuda.synchronize()
    for i in range(m):
        want, ws = ref.quantize_blocks(x[i].double().numpy())
        assert np.array_equal(s[i, :, :cb].cpu().numpy(), ws) and _same(_values(q[i]), want)
        if turned:
            assert np.array_equal(st[i, :, :rb].cpu().numpy(), ws.T) and _same(_values(qt[i]), want.T)
    assert (qb[:, rows:] == SENTINEL).all() and (qb[:, :, cols:] == SENTINEL).all() and (s[:, :, cb:] == SENTINEL).all()
    if turned:
        assert (qtb[:, cols:] == SENTINEL).all() and (qtb[:, :, rows:] == SENTINEL).all() and (st[:, :, rb:] == SENTINEL).all()
    else:
        assert (qtb == SENTINEL).all() and (st == SENTINEL).all()


@pytest.mark.parametrize("T,E,k,score,renorm", [(40001, 64, 8, "softmax", False), (20003, 256, 8, "sigmoid", True), (19001, 60, 17, "softmax", True)])
def test_route_backward_of_several_tokens_a_warp(T, E, k, score, renorm):
    from paper_2609_04609_b200 import ciera

    logits = _logits(T, E, "fp32", 3)
    logits[T - 2, : E // 2] = float("-inf")
    g = torch.Generator().manual_seed(4)
    experts = torch.rand(T, E, generator=g).topk(k, 1).indices.int()
    experts[5::1000, 1] = -1
    experts[7::1000, 0] = experts[7::1000, 2]  # the same index twice
    dw = torch.randn(T, k, generator=g)
    out = torch.full((T + 1, E), 7.0, device=DEV)
    ciera.route_backward(_config(E, k, score, renorm=renorm, scale=2.0), logits.to(DEV), experts.to(DEV), dw.to(DEV), out[:T])
    torch.cuda.synchronize()
    assert (out[T] == 7.0).all()
    # the formula in 64 bits on the GPU
    x, at, d = logits.to(DEV).double(), experts.to(DEV).long(), dw.to(DEV).double()
    s = x.softmax(1) if score == "softmax" else x.sigmoid()
    some = at >= 0
    sk = s.gather(1, at.clamp(min=0)) * some
    d = d * some * 2.0
    total = sk.sum(1, keepdim=True)
    if renorm:
        d = (d - (d * sk).sum(1, keepdim=True) / total) / total * some
    ds = torch.zeros_like(s).scatter_add_(1, at.clamp(min=0), d)
    want = ds * s * (1 - s) if score == "sigmoid" else s * (ds - (ds * s).sum(1, keepdim=True))
    # as in test_gpu_route: s is off by (E + 8) steps of 32 bits, ds and the sum of ds s by (E + k + 16) steps of their largest term
    term = 2.0 * dw.abs().amax(1, keepdim=True).to(DEV).double()
    if renorm:
        term = 2 * term / total
    tol = 2 * (E + k + 24) * 2.0**-24 * s * term * (k + 1) + 2.0**-24 * want.abs() + 1e-37
    assert ((out[:T].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("T,k,cols,dtype", [(12001, 2, 2048, "bf16"), (70001, 3, 37, "fp32"), (30001, 8, 130, "fp16")])
def test_weighted_sums_of_more_work_than_threads(T, k, cols, dtype):
    from paper_2609_04609_b200 import ciera

    g = torch.Generator(device=DEV).manual_seed(T)
    n = T * k + 5
    dt = DTYPES[dtype]
    rows = torch.randn(n, cols, generator=g, device=DEV).to(dt)
    at = torch.randperm(n, generator=g, device=DEV)[: T * k].view(T, k).int()
    at[3::50, 0] = -1
    at[4] = n  # outside
    w = torch.rand(T, k, generator=g, device=DEV)
    out = torch.full((T + 1, cols), 9.0, dtype=dt, device=DEV)
    ciera.expert_combine(rows, at, w, out[:T])
    assert (out[T] == 9.0).all()
    some = (at >= 0) & (at < n)
    index = torch.where(some, at, 0).long()
    step = torch.finfo(dt).eps / 2
    small = 6e-8 if dtype == "fp16" else 0.0
    want, size = torch.zeros(T, cols, dtype=torch.float64, device=DEV), torch.zeros(T, cols, dtype=torch.float64, device=DEV)
    for j in range(k):
        term = rows[index[:, j]].double() * (w[:, j] * some[:, j]).double()[:, None]
        want += term
        size += term.abs()
    assert ((out[:T].double() - want).abs() <= (k + 1) * 2.0**-24 * size + step * want.abs() + small).all()
    dout = torch.randn(T, cols, generator=g, device=DEV).to(dt)
    dw = torch.full((T + 1, k), 9.0, device=DEV)
    drows = torch.full((n, cols), 9.0, dtype=dt, device=DEV)
    ciera.expert_combine_backward(dout, rows, at, w, dw[:T], drows)
    torch.cuda.synchronize()
    assert (dw[T] == 9.0).all()
    named = torch.zeros(n, dtype=torch.bool, device=DEV)
    named[index[some]] = True
    assert (drows[~named] == 9.0).all()
    for j in range(k):
        r, d, ok = rows[index[:, j]].double(), dout.double(), some[:, j]
        dot, dot_size = (r * d).sum(1) * ok, (r * d).abs().sum(1) * ok
        assert ((dw[:T, j].double() - dot).abs() <= (cols + 2) * 2.0**-24 * dot_size).all()
        grad = (d * w[:, j].double()[:, None])[ok]
        assert ((drows[index[ok, j]].double() - grad).abs() <= (step + 2.0**-23) * grad.abs() + small).all()
