"""Slots in the order of the experts, and the weighted sum of a token's rows with its gradients."""
import numpy as np
import pytest
import torch

from tests import moe_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _ids(T, k, E, seed, skew=0.5, dropped=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = (torch.randn(T, E, generator=g) + skew * torch.randn(E, generator=g)).topk(k, 1).indices.int()
    return torch.where(torch.rand(T, k, generator=g) < dropped, torch.full_like(ids, -1), ids)


def _run(ids, E):
    from paper_2609_04609_b200 import ciera

    n = ids.numel()
    cap = ciera.expert_rows_capacity(n, E)
    starts = torch.full((E + 2,), -9, dtype=torch.int32, device=DEV)
    counts = torch.full((E + 1,), -9, dtype=torch.int32, device=DEV)
    ros = torch.full((n + 1,), -9, dtype=torch.int32, device=DEV)
    sor = torch.full((cap + 1,), -9, dtype=torch.int32, device=DEV)
    ws = torch.full((ciera.expert_layout_workspace_bytes(n, E),), 0xAB, dtype=torch.uint8, device=DEV)
    ciera.expert_layout(ids.to(DEV), E, starts[: E + 1], counts[:E], ros[:n].view(ids.shape), sor[:cap], ws)
    torch.cuda.synchronize()
    assert starts[E + 1] == -9 and counts[E] == -9 and ros[n] == -9 and sor[cap] == -9
    return starts[: E + 1].tolist(), counts[:E].tolist(), ros[:n].tolist(), sor[:cap].tolist()


@pytest.mark.parametrize("T,k,E,skew,dropped", [
    (1, 8, 64, 0.5, 0.0), (1, 1, 1, 0.0, 0.0), (33, 8, 64, 0.5, 0.2), (128, 1, 4, 0.0, 0.0), (255, 8, 8, 0.0, 0.0),
    (257, 8, 300, 2.0, 0.0), (256, 8, 1024, 1.0, 0.5), (513, 4, 1000, 0.0, 0.0), (3001, 8, 64, 1.5, 0.1), (20000, 6, 160, 0.8, 0.0),
    (2048, 1, 2, 9.0, 0.0), (2049, 1, 2, 9.0, 0.0),
])
def test_layout_equals_the_definition(T, k, E, skew, dropped):
    ids = _ids(T, k, E, T + E, skew, dropped)
    starts, counts, ros, sor = _run(ids, E)
    w_starts, w_counts, w_ros, w_sor = ref.layout(ids, E)
    assert starts == w_starts and counts == w_counts and ros == w_ros
    assert sor[: starts[-1]] == [w_sor[r] for r in range(starts[-1])]
    assert all(v == -9 for v in sor[starts[-1] :])  # rows behind the last segment are left as they were


def test_layout_without_slots_and_with_none_taken():
    starts, counts, ros, sor = _run(torch.zeros(0, 8, dtype=torch.int32), 5)
    assert starts == [0] * 6 and counts == [0] * 5
    for T in (9, 3000):
        ids = torch.full((T, 2), -1, dtype=torch.int32)
        ids[0, 1], ids[1, 0] = 5, 2**31 - 1  # outside
        starts, counts, ros, sor = _run(ids, 5)
        assert starts == [0] * 6 and counts == [0] * 5 and ros == [-1] * (2 * T) and set(sor) <= {-9}


def test_layout_of_one_expert_many_times():
    ids = torch.full((4000, 2), 3, dtype=torch.int32)  # the same index twice in a token, all in one segment
    starts, counts, ros, sor = _run(ids, 64)
    assert counts[3] == 8000 and sum(counts) == 8000 and ros == list(range(8000))


def test_capacity_is_enough_for_every_spread():
    from paper_2609_04609_b200 import ciera

    for n in (0, 1, 5, 127, 128, 129, 1000, 100000):
        for E in (1, 2, 64, 1024):
            # worst: as many experts as possible hold one slot more than a multiple of 128
            some = min(n, E)
            left = n - some
            worst = 128 * (some + left // 128)
            assert ciera.expert_rows_capacity(n, E) >= worst


@pytest.mark.parametrize("T,k,H,dtype,weighted,dropped", [
    (1, 8, 2048, "bf16", True, 0.0), (1, 1, 1, "fp32", False, 0.0), (33, 8, 2050, "bf16", True, 0.1), (100, 3, 77, "fp16", True, 0.0),
    (300, 32, 64, "fp32", False, 0.3), (1023, 2, 1028, "fp16", False, 0.0), (77, 8, 515, "fp32", True, 0.0),
])
def test_combine_and_its_gradients(T, k, H, dtype, weighted, dropped):
    from paper_2609_04609_b200 import ciera

    dt, E = DTYPES[dtype], 64
    ids = _ids(T, k, E, T + H, 0.5, dropped)
    if T > 2:
        ids[2] = -1  # a token without rows
    starts, counts, ros, sor = ref.layout(ids, E)
    n_rows = max(starts[-1], 1)
    at = torch.tensor(ros, dtype=torch.int32).view(T, k)
    if T > 5:
        at[5, 0] = n_rows  # outside: passed over
    g = torch.Generator().manual_seed(H)
    rows = torch.randn(n_rows, H, generator=g).to(dt)
    rows[[r for r in range(starts[-1]) if sor[r] < 0]] = float("nan")  # rows that no slot names are not read
    w = torch.rand(T, k, generator=g) if weighted else None
    dout = torch.randn(T, H, generator=g).to(dt)

    def wide(t, fill):
        buf = torch.full((t.shape[0], t.shape[1] + (3 if T % 2 else 0)), fill, dtype=t.dtype, device=DEV)
        buf[:, : t.shape[1]] = t.to(DEV)
        return buf, buf[:, : t.shape[1]]

    _, d_rows = wide(rows, 3.0)
    _, d_dout = wide(dout, 3.0)
    out_all, out = wide(torch.zeros(T, H, dtype=dt), 5.0)
    dr_all, dr = wide(torch.full((n_rows, H), 7.0, dtype=dt), 7.0)
    dwt = torch.zeros(T, k, device=DEV)
    dw_ = None if w is None else w.to(DEV)
    ciera.expert_combine(d_rows, at.to(DEV), dw_, out)
    ciera.expert_combine_backward(d_dout, d_rows, at.to(DEV), dw_, dwt, dr)
    torch.cuda.synchronize()
    assert (out_all[:, H:] == 5.0).all() and (dr_all[:, H:] == 7.0).all()
    live = (at >= 0) & (at < n_rows)
    y = rows.double()[at.long().clamp(0, n_rows - 1)]
    y[~live] = 0.0
    w64 = torch.ones(T, k, dtype=torch.float64) if w is None else w.double()
    w64 = w64 * live
    step = torch.finfo(dt).eps / 2
    terms = w64[:, :, None] * y
    want, size = terms.sum(1), terms.abs().sum(1)
    # k products and k additions in 32 bits, one rounding to the type
    assert ((out.double().cpu() - want).abs() <= (k + 2) * 2.0**-24 * size + step * want.abs() + 1e-7 * (dtype == "fp16")).all()
    prod = dout.double()[:, None] * y
    # H products and additions in 32 bits, in any order
    assert ((dwt.double().cpu() - prod.sum(2)).abs() <= (H + 2) * 2.0**-24 * prod.abs().sum(2)).all()
    want_rows = torch.full((n_rows, H), 7.0, dtype=torch.float64)
    want_rows[at[live].long()] = (w64[:, :, None] * dout.double()[:, None])[live]
    assert ((dr.double().cpu() - want_rows).abs() <= (step + 2.0**-24) * want_rows.abs() + 1e-7 * (dtype == "fp16")).all()
    # without the rows' gradient
    again = torch.zeros_like(dwt)
    ciera.expert_combine_backward(d_dout, d_rows, at.to(DEV), dw_, again)
    assert torch.equal(again, dwt)


def test_layout_and_combine_in_two_graphs():
    """Two captured graphs, each with its own workspace, replayed on two streams at the same time."""
    from paper_2609_04609_b200 import ciera

    T, k, E, H = 3000, 8, 64, 256
    n = T * k
    cap = ciera.expert_rows_capacity(n, E)
    sides = []
    for s in range(2):
        st = dict(ids=_ids(T, k, E, s).to(DEV), starts=torch.zeros(E + 1, dtype=torch.int32, device=DEV),
                  counts=torch.zeros(E, dtype=torch.int32, device=DEV), ros=torch.zeros(T, k, dtype=torch.int32, device=DEV),
                  sor=torch.zeros(cap, dtype=torch.int32, device=DEV),
                  ws=torch.zeros(ciera.expert_layout_workspace_bytes(n, E), dtype=torch.uint8, device=DEV),
                  rows=torch.randn(cap, H, device=DEV), out=torch.zeros(T, H, device=DEV), stream=torch.cuda.Stream())

        def call(st=st):
            ciera.expert_layout(st["ids"], E, st["starts"], st["counts"], st["ros"], st["sor"], st["ws"])
            ciera.expert_combine(st["rows"], st["ros"], None, st["out"])

        call()
        torch.cuda.synchronize()
        st["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(st["graph"]):
            call()
        sides.append(st)
    for rnd in range(3):
        for s, st in enumerate(sides):
            st["ids"].copy_(_ids(T, k, E, 10 * rnd + s, dropped=0.1))
        torch.cuda.synchronize()
        for st in sides:
            with torch.cuda.stream(st["stream"]):
                st["graph"].replay()
        torch.cuda.synchronize()
        for st in sides:
            _, counts, ros, _ = ref.layout(st["ids"].cpu(), E)
            assert st["ros"].reshape(-1).tolist() == ros and st["counts"].tolist() == counts
            y = st["rows"].double()[st["ros"].long().clamp(min=0)] * (st["ros"] >= 0)[:, :, None]
            assert ((st["out"].double() - y.sum(1)).abs() <= 10 * 2.0**-24 * y.abs().sum(1)).all()
