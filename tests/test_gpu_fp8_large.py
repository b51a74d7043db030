"""Products of sizes at which a pair of blocks has tiles of 256 rows and several of them (at least 74 tiles of 256 x 256)."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref
from tests.test_gpu_fp8 import DTYPES, _close, _matrices, _operand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("b_rows", [False, True])
@pytest.mark.parametrize("m,n,k,out", [
    (2500, 2000, 500, "bf16"), (4096, 2048, 128, "fp32"), (2433, 2049, 1290, "fp32"), (5000, 4100, 260, "fp16"), (20000, 250, 130, "bf16"),
])
def test_dense_product_of_many_tiles(b_rows, m, n, k, out):
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
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ciera.fp8_matmul(a, sa, b, sb, o[:m, :n], status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert (o[m] == 9.0).all() and (o[:, n:] == 9.0).all()
    assert _close(o[:m, :n], ref.operand_values(a, sa), vb)


# segments that end in a tile's first and second half, empty ones, one of many tiles
SEGMENTS = [[384, 128, 0, 640, 256, 1024, 128], [0, 2688, 0, 0], [128] * 30 + [896] * 3, [2560 + 128, 256, 384]]


@pytest.mark.parametrize("segments", SEGMENTS, ids=lambda s: "-".join(map(str, s))[:24])
@pytest.mark.parametrize("n,k,out", [(2048, 384, "bf16"), (2049, 1030, "fp32"), (2500, 128, "fp16")])
def test_product_by_segments_of_rows_of_many_tiles(segments, n, k, out):
    from paper_2609_04609_b200 import ciera

    E = len(segments)
    starts = torch.tensor([0] + list(np.cumsum(segments)), dtype=torch.int32, device=DEV)
    used = int(starts[-1])
    rows = used + 130
    a, sa = _operand(rows, k, k)
    a.view(torch.uint8)[used:] = 0x7F
    if out == "fp16":
        sa[:, :rows] -= 10
    b, sb = _matrices(E, n, k, n)
    o = torch.full((rows, n), 9.0, dtype=DTYPES[out], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ciera.fp8_matmul(a, sa, b, sb, o, starts, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    va, vb = ref.operand_values(a, sa), ref.matrix_values(b, sb)
    for e in range(E):
        lo, hi = int(starts[e]), int(starts[e + 1])
        assert hi == lo or _close(o[lo:hi], va[lo:hi], vb[e]), f"expert {e}"
    assert (o[used:] == 9.0).all()


@pytest.mark.parametrize("m,n,out", [(600, 1000, "fp32"), (513, 2050, "bf16"), (256, 2500, "fp32"), (130, 5000, "fp32")])
def test_product_by_segments_of_the_contraction_of_many_tiles(m, n, out):
    from paper_2609_04609_b200 import ciera

    segments = [256, 0, 384, 128, 1280, 0, 128, 640]
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
        assert (o[e] == 0).all() if hi == lo else _close(o[e], va[:, lo:hi], vb[:, lo:hi]), f"expert {e}"


def test_launches_behind_one_another_give_the_same_bits():
    """Many short launches without a pause: blocks of one leave while those of the next come, from one and from two streams."""
    from paper_2609_04609_b200 import ciera

    segments = [384, 128, 0, 640, 256, 1024, 128]
    n, k = 2048, 256
    starts = torch.tensor([0] + list(np.cumsum(segments)), dtype=torch.int32, device=DEV)
    rows = int(starts[-1])
    a, sa = _operand(rows, k, 1)
    b, sb = _matrices(len(segments), n, k, 2)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = torch.zeros(rows, n, device=DEV)
    ciera.fp8_matmul(a, sa, b, sb, want, starts, status=status)
    va, vb = ref.operand_values(a, sa), ref.matrix_values(b, sb)
    for e in range(len(segments)):
        lo, hi = int(starts[e]), int(starts[e + 1])
        assert hi == lo or _close(want[lo:hi], va[lo:hi], vb[e])
    outs, streams = [torch.zeros(16, rows, n, device=DEV) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(16):
        for s, o in zip(streams, outs):
            ciera.fp8_matmul(a, sa, b, sb, o[i], starts, status=status, stream=s)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert all(torch.equal(o, want.expand_as(o)) for o in outs)
