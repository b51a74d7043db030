"""Layouts of many chunks of slots, where their counts are added up in a launch of their own."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CHUNK = 4096


def _check(ids, E):
    from paper_2609_04609_b200 import ciera

    n = ids.numel()
    cap = ciera.expert_rows_capacity(n, E)
    i32 = dict(dtype=torch.int32, device=DEV)
    starts, counts = torch.full((E + 1,), -9, **i32), torch.full((E,), -9, **i32)
    ros, sor = torch.full((n + 1,), -9, **i32), torch.full((cap + 1,), -9, **i32)
    bytes_ = ciera.expert_layout_workspace_bytes(n, E)
    ws = torch.full((bytes_ + 64,), 0xAB, dtype=torch.uint8, device=DEV)
    for _ in range(2):  # (any contents of the workspace)
        ciera.expert_layout(ids, E, starts, counts, ros[:n].view(ids.shape), sor[:cap], ws[:bytes_])
    torch.cuda.synchronize()
    assert (ws[bytes_:] == 0xAB).all() and ros[n] == -9 and sor[cap] == -9
    flat = ids.reshape(-1).long()
    some = (flat >= 0) & (flat < E)
    key = torch.where(some, flat, E)
    want = torch.bincount(key, minlength=E + 1)[:E]
    assert torch.equal(counts.long(), want)
    first = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    first[1:] = ((want + 127) // 128 * 128).cumsum(0)
    assert torch.equal(starts.long(), first)
    order = torch.sort(key, stable=True).indices  # slots in the order of their experts, those without one last
    before = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    before[1:] = want.cumsum(0)
    rank = torch.empty_like(order)
    rank[order] = torch.arange(n, device=DEV)
    row = torch.where(some, first[key] + rank - before[key], -1)
    assert torch.equal(ros[:n].long(), row)
    slots = torch.full((cap,), -9, dtype=torch.int64, device=DEV)
    slots[: int(first[E])] = -1
    slots[row[some]] = torch.arange(n, device=DEV)[some]
    assert torch.equal(sor[:cap].long(), slots)


@pytest.mark.parametrize("E", [1, 7, 64, 300, 1024])
@pytest.mark.parametrize("n", [254 * CHUNK + 5, 255 * CHUNK, 255 * CHUNK + 1, 256 * CHUNK, 300 * CHUNK + 77])
def test_layout_around_the_change(n, E):
    g = torch.Generator(device=DEV).manual_seed(n + E)
    ids = (torch.randn(n, generator=g, device=DEV).abs() * E / 2.5).int()  # (some beyond the last expert)
    ids[:: 97] = -1
    _check(ids, E)


def test_layout_of_very_many_slots():
    g = torch.Generator(device=DEV).manual_seed(1)
    ids = torch.randint(0, 512, (1 << 22, 8), generator=g, dtype=torch.int32, device=DEV)  # 8192 chunks
    _check(ids, 512)


def test_layout_of_many_chunks_from_a_graph():
    from paper_2609_04609_b200 import ciera

    E, n = 64, 260 * CHUNK
    ids = torch.zeros(n, dtype=torch.int32, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    starts, counts, ros = torch.zeros(E + 1, **i32), torch.zeros(E, **i32), torch.zeros(n, **i32)
    sor = torch.zeros(ciera.expert_rows_capacity(n, E), **i32)
    ws = torch.zeros(ciera.expert_layout_workspace_bytes(n, E), dtype=torch.uint8, device=DEV)
    ciera.expert_layout(ids, E, starts, counts, ros, sor, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ciera.expert_layout(ids, E, starts, counts, ros, sor, ws)
    for seed in (1, 2):
        ids.copy_(torch.randint(0, E, (n,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32))
        graph.replay()
        got = [t.clone() for t in (starts, counts, ros)]
        ciera.expert_layout(ids, E, starts, counts, ros, sor, ws)
        assert all(torch.equal(a, b) for a, b in zip(got, (starts, counts, ros)))
        assert torch.equal(counts.long(), torch.bincount(ids.long(), minlength=E))
