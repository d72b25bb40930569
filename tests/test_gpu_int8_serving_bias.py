"""A routing bias in the serving loop, with and without a rule beside it."""
import pytest
import torch

from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.paged_serving import PagedServer, Request
from paper_2605_23296_amd.workloads import make_weights
from tests.test_gpu_int8_serving import LAYERS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("int8", [False, True])
def test_a_bias_without_a_rule_is_the_own_rules(int8):
    cfg, gen = LAYERS["routed_bf16"], torch.Generator().manual_seed(3)
    w = {k: v.cuda() for k, v in make_weights(cfg, gen).items()}
    x = torch.randn((50, cfg.d_model), generator=gen).bfloat16().cuda()
    bias = torch.zeros(16).cuda()
    bias[[3, 5, 9, 15]] = 10.0          # scores are 1 at most: these four are everybody's experts

    def run(**kw):
        server = PagedServer(cfg, w, 1, 8, 16, 64, max_len=64, int8=int8, **kw)
        r = Request(x, None)
        assert server.submit(r)
        while server.step():
            pass
        return torch.cat(r.out)
    alone = run(route_bias=bias)
    assert torch.equal(alone, run(route=B.RouteRule(), route_bias=bias))
    assert not torch.equal(alone, run())
