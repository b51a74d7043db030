"""The operators behind the gather called from several host threads at once."""
import threading

import pytest
import torch

from tests import moe_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_layouts_of_different_widths_from_several_threads():
    from paper_2609_04609_b200 import ciera

    torch.zeros(1, device=DEV)
    problems = []

    def work(E, seed):
        try:
            stream = torch.cuda.Stream()
            g = torch.Generator().manual_seed(seed)
            ids = torch.rand(40, E, generator=g).topk(4, 1).indices.int()
            want, _, ros, _ = ref.layout(ids, E)
            with torch.cuda.stream(stream):
                dev = ids.to(DEV)
                cap = ciera.expert_rows_capacity(ids.numel(), E)
                i32 = dict(dtype=torch.int32, device=DEV)
                starts, counts, rows, slots = torch.zeros(E + 1, **i32), torch.zeros(E, **i32), torch.zeros_like(dev), torch.zeros(cap, **i32)
                ws = torch.zeros(ciera.expert_layout_workspace_bytes(ids.numel(), E), dtype=torch.uint8, device=DEV)
                for _ in range(4000):
                    ciera.expert_layout(dev, E, starts, counts, rows, slots, ws)
            stream.synchronize()
            assert starts.tolist() == want and rows.reshape(-1).tolist() == ros
        except BaseException as e:  # noqa: BLE001
            problems.append(f"{E} experts: {e!r}")

    threads = [threading.Thread(target=work, args=(E, i)) for i, E in enumerate((1024, 700, 900, 1000))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not problems, problems
