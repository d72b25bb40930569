"""The serving loop's own bookkeeping, on the host: no call reaches the GPU here."""
import torch

from paper_2605_23296_amd.paged_serving import PagedServer, Request
from paper_2605_23296_amd.workloads import LayerConfig, make_weights

CFG = LayerConfig(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=256, dtype="bf16")


def server(**over):
    kw = dict(n_slots=2, n_pages=4, page_rows=16, max_rows=32, max_len=64)
    return PagedServer(CFG, make_weights(CFG, torch.Generator().manual_seed(1)), device="cpu", **dict(kw, **over))


def rows(n):
    return torch.zeros((n, CFG.d_model), dtype=torch.bfloat16)


def test_a_request_without_rows_is_done_at_once():
    s = server()
    for r in (Request(rows(0), None), Request(rows(0), rows(0)), Request(rows(0), None)):     # more of them than there are slots
        assert s.submit(r) and r.out == []
    assert s.slots == [None, None] and s.free == 4 and s.step() == 0
    assert s.submit(Request(rows(0), rows(3)))       # rows of decode steps alone are a request like others
    assert s.slots[0] is not None
