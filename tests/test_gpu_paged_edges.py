"""Paged cache in 8 bits at the edges of what its calls accept: requests without cached rows beside pages that hold anything."""
import pytest
import torch

from paper_2605_23296_amd import binding as B
from tests.test_gpu_paged import ATTN_LAYERS, IDS, check_attn, handle, queries, random_cache, run_attn

pytestmark = pytest.mark.gpu


def with_nobodys_page_0(kv, ref, table):
    """The same cache behind one more page that no request owns, full of NaN codes and NaN scales."""
    def behind(x, fill):
        return torch.cat([torch.full_like(x[:1], fill), x])
    kv = B.PagedKV(kv.layer, behind(kv.k, 0x7F), behind(kv.v, 0x7F), behind(kv.k_scale, 255), behind(kv.v_scale, 255), kv.table + (kv.table >= 0).int())
    return kv


@pytest.mark.parametrize("lc", ATTN_LAYERS, ids=IDS)
@pytest.mark.parametrize("n_new,lens", [([1, 1, 1], [0, 300, 0]), ([4, 2, 1], [0, 40, 0]), ([1, 4, 1, 90, 2], [0, 0, 300, 100, 0])],
                         ids=["single_tokens", "a_few_rows", "beside_a_prompt"])
@pytest.mark.parametrize("entry", [-1, 0])
def test_requests_without_cached_rows_give_zeros(lc, n_new, lens, entry):
    """As the plan leaves a request that it refused: rows in the batch, no cached ones, and a table row that names nothing or a page
    of somebody else's, here one whose codes and scales are NaN."""
    kv, ref, table = random_cache(lc, lens, 32, 21)
    kv = with_nobodys_page_0(kv, ref, table)
    for i, L in enumerate(lens):
        if L == 0:
            kv.table[i].fill_(entry)
    q, lay = queries(lc, sum(n_new), 21), handle(lc)
    o = run_attn(lay, kv, q, n_new, lens)
    check_attn(lc, q, o, n_new, lens, ref, table)
    for rows, L in zip(torch.split(o, n_new), lens):
        assert L > 0 or (rows == 0).all()
