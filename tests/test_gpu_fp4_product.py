"""Products of 4-bit operands against 64 bits."""
import numpy as np
import pytest
import torch

from tests import fp4_reference as f4
from tests.test_gpu_fp8 import DTYPES, _layout

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _close(out, a, b):
    """k terms added in 32 bits in any order, and one rounding to the result's type."""
    k = a.shape[1]
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    step = torch.finfo(out.dtype).eps / 2
    tol = (k + 2) * 2.0**-24 * size + step * np.abs(want) + (2.0**-25 if out.dtype == torch.float16 else 0)
    return bool((np.abs(out.double().cpu().numpy() - want) <= tol).all())


def _operand(rows, cols, seed, spread=8):
    codes, s = f4.random_operand(rows, cols, seed, spread)
    return (*f4.operand_tensors(codes, s, DEV), f4.values(codes, s))


@pytest.mark.parametrize("m,n,k,dtype", [
    (1, 1, 1, "fp32"), (1, 256, 64, "bf16"), (128, 128, 128, "fp32"), (129, 257, 65, "bf16"), (300, 100, 511, "fp32"), (64, 300, 640, "fp16"),
    (256, 512, 1024, "fp32"), (513, 129, 96, "bf16"), (1000, 1111, 777, "fp32"), (5, 2048, 2048, "bf16"), (7, 33, 2305, "fp32"),
])
def test_dense(m, n, k, dtype):
    from paper_2609_04609_b200 import ciera

    a, a_s, av = _operand(m, k, m + k)
    b, b_s, bv = _operand(n, k, n + k + 1)
    out = torch.full((m, n + 2), 7.0, dtype=DTYPES[dtype], device=DEV)
    ciera.fp4_matmul(a, a_s, b, b_s, out[:, :n])
    assert _close(out[:, :n], av, bv)
    assert (out[:, n:] == 7.0).all()


def test_many_tiles_take_both_sums_and_all_stages():
    from paper_2609_04609_b200 import ciera

    m, n, k = 4100, 8200, 1540
    a, a_s, av = _operand(m, k, 3)
    b, b_s, bv = _operand(n, k, 4)
    out = torch.zeros(m, n, dtype=torch.float32, device=DEV)
    ciera.fp4_matmul(a, a_s, b, b_s, out)
    ad, bd = torch.from_numpy(av).to(DEV), torch.from_numpy(bv).to(DEV)
    size = ad.abs() @ bd.abs().T
    assert ((out.double() - ad @ bd.T).abs() <= (k + 2) * 2.0**-24 * size).all()
    again = torch.zeros_like(out)
    ciera.fp4_matmul(a, a_s, b, b_s, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("T,top_k,E,n,k,dtype", [
    (1, 2, 4, 256, 256, "bf16"), (77, 3, 5, 130, 200, "fp32"), (400, 2, 3, 384, 96, "bf16"), (3, 1, 64, 300, 577, "fp16"), (1500, 2, 7, 520, 160, "fp32"),
])
def test_rows_by_segments(T, top_k, E, n, k, dtype):
    from paper_2609_04609_b200 import ciera

    starts, slot, cap = _layout(T, top_k, E, T)
    used = int(starts[-1])
    codes, s = f4.random_operand(cap, k, T)
    codes[:used][slot[:used].numpy() < 0] = 0
    s[used:] = 255  # behind the last segment: nothing that counts
    a, a_s = f4.operand_tensors(codes, s, DEV)
    av = f4.values(codes, s)
    parts = [f4.random_operand(n, k, 100 + e) for e in range(E)]
    bs = [f4.operand_tensors(*p, DEV) for p in parts]
    line = bs[0][0].shape[1]
    b = torch.zeros(E, n, -(-line // 16) * 16, dtype=torch.uint8, device=DEV)[:, :, :line]
    for e in range(E):
        b[e] = bs[e][0]
    b_s = torch.stack([x[1] for x in bs])
    out = torch.full((cap, n), 7.0, dtype=DTYPES[dtype], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ciera.fp4_matmul(a, a_s, b, b_s, out, starts.to(DEV), status)
    assert int(status) == 0 and (out[used:] == 7.0).all()
    for e in range(E):
        lo, hi = int(starts[e]), int(starts[e + 1])
        if lo < hi:
            assert _close(out[lo:hi], av[lo:hi], f4.values(*parts[e]))


@pytest.mark.parametrize("bad", [[0, 128, 100, 256], [0, 256, 128, 384], [128, 256, 256, 384], [0, 128, 256, 512], [0, -128, 128, 256]])
def test_a_table_that_does_not_rise_is_reported(bad):
    from paper_2609_04609_b200 import ciera

    a, a_s, _ = _operand(384, 64, 1)
    b, b_s, _ = _operand(3 * 128, 64, 2)
    out = torch.full((384, 128), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ciera.fp4_matmul(a, a_s, b.reshape(3, 128, 32), b_s[:, None], out, torch.tensor(bad, dtype=torch.int32, device=DEV), status)
    assert int(status) == ciera.ERR_CORRUPT and (out == 7.0).all()


def test_a_group_that_is_not_finite_reaches_its_own_row_and_column():
    from paper_2609_04609_b200 import ciera

    m, n, k = 200, 300, 320
    codes, s = f4.random_operand(m, k, 5)
    s[17, 4] = 255
    a, a_s = f4.operand_tensors(codes, s, DEV)
    bc, bsc = f4.random_operand(n, k, 6)
    bsc[123, 9] = 255
    b, b_s = f4.operand_tensors(bc, bsc, DEV)
    out = torch.zeros(m, n, device=DEV)
    ciera.fp4_matmul(a, a_s, b, b_s, out)
    want = np.zeros((m, n), bool)
    want[17], want[:, 123] = True, True
    assert np.array_equal(torch.isnan(out).cpu().numpy(), want)


def test_scales_over_their_whole_range():
    """One group, one term: the product of two powers of two anywhere, rounded once."""
    from paper_2609_04609_b200 import ciera

    codes = np.full((254, 32), 0)
    codes[:, 0] = 2  # 1.0
    s = np.arange(1, 255)[:, None]
    a, a_s = f4.operand_tensors(codes, s, DEV)
    out = torch.zeros(254, 254, device=DEV)
    ciera.fp4_matmul(a, a_s, a, a_s, out)
    e = s - 127.0
    want = torch.from_numpy(2.0 ** (e + e.T)).float()
    normal = (want >= 2.0**-126) & (want < float("inf"))  # (below that the sums may be flushed)
    assert torch.equal(out.cpu()[normal], want[normal])
    assert (out.cpu()[want < 2.0**-126] <= 2.0**-126).all() and torch.isinf(out.cpu()[torch.isinf(want)]).all()


def test_captured_and_replayed_with_other_segments():
    from paper_2609_04609_b200 import ciera

    a, a_s, av = _operand(512, 256, 1)
    parts = [f4.random_operand(200, 256, 9 + e) for e in range(2)]
    ts = [f4.operand_tensors(*p, DEV) for p in parts]
    b, b_s = torch.stack([t[0] for t in ts]), torch.stack([t[1] for t in ts])
    starts = torch.tensor([0, 128, 256], dtype=torch.int32, device=DEV)
    out = torch.full((512, 200), 7.0, device=DEV)
    ciera.fp4_matmul(a, a_s, b, b_s, out, starts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ciera.fp4_matmul(a, a_s, b, b_s, out, starts)
    starts.copy_(torch.tensor([0, 384, 512]))
    out.fill_(7.0)
    graph.replay()
    assert _close(out[:384], av[:384], f4.values(*parts[0])) and _close(out[384:], av[384:], f4.values(*parts[1]))
