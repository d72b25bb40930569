"""The serving loop over the paged cache: every row of every request against the layer in 64 bits over the rows that the
cache holds, while requests arrive, prefill in chunks, decode, leave and hand their pages on."""
import numpy as np
import pytest
import torch

from oracle import layer as O
from oracle import paged8 as P8
from paper_2605_23296_amd.paged_serving import PagedServer, Request
from paper_2605_23296_amd.workloads import LayerConfig, make_weights, to_numpy_f64
from tests.util import BF16_VEC_TOL, FP32_TOL, rel_err, vec_rel_err

pytestmark = pytest.mark.gpu

LAYERS = {
    "dense_bf16": LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, ffn_dim=1024, rope_theta=500000.0, dtype="bf16"),
    "dense_bf16_128": LayerConfig(d_model=640, n_q_heads=5, n_kv_heads=5, head_dim=128, ffn_dim=512, dtype="bf16"),
    "dense_fp32": LayerConfig(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=512, dtype="fp32"),
    "routed_fp32": LayerConfig(d_model=256, n_q_heads=4, n_kv_heads=1, head_dim=64, ffn_dim=128, n_experts=8, top_k=2, dtype="fp32"),
}


@pytest.mark.parametrize("name", LAYERS)
@pytest.mark.parametrize("page_rows,max_rows,n_pages", [(16, 96, 24), (64, 300, 8)])
def test_rows_of_a_continuous_batch(name, page_rows, max_rows, n_pages):
    cfg = LAYERS[name]
    gen = torch.Generator().manual_seed(7)
    w = make_weights(cfg, gen, gain_jitter=True)
    ref = O.Layer(cfg.as_dict(), {k: to_numpy_f64(v) for k, v in w.items()})
    server = PagedServer(cfg, {k: v.cuda() for k, v in w.items()}, 3, n_pages, page_rows, max_rows, max_len=320)
    dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32

    def rows(n):
        return torch.randn((n, cfg.d_model), generator=gen).to(dt).cuda()
    waiting = [Request(rows(L), rows(S)) for L, S in ((150, 5), (1, 3), (17, 9), (64, 2), (200, 1), (33, 20), (16, 16))]
    every, total, steps = list(waiting), sum(r.rows.shape[0] for r in waiting), 0
    done = 0
    while True:
        while waiting and server.submit(waiting[0]):
            waiting.pop(0)
        before = [(r, None if r is None else r.done) for r in server.slots]
        ran = server.step()
        if ran == 0 and not waiting:
            break
        done, steps = done + ran, steps + 1
        assert int(server.st.n_refused) == 0
        for i, (r, d0) in enumerate(before):
            if r is None or r.done == d0:
                continue
            K, V = (to_numpy_f64(t) for t in server.kv.rows(i, r.done))
            x = to_numpy_f64(r.rows[d0:r.done])
            q, k, v = ref.qkv(x, np.arange(d0, r.done))
            h = x + P8.attend(q, K, V).reshape(len(x), -1) @ ref.w["w_o"].T
            y = ref.ffn(h)[0]
            got = to_numpy_f64(r.out[-1])
            if cfg.dtype == "bf16":
                assert vec_rel_err(got, y) < BF16_VEC_TOL, (i, d0)
            else:
                assert rel_err(got, y) < FP32_TOL, (i, d0)
            # a code is within 2^-4 of its value, that within the projections' own error
            assert vec_rel_err(K[d0:], k) < 2.0 ** -4 + 1e-2 and vec_rel_err(V[d0:], v) < 2.0 ** -4 + 1e-2
    assert done == total and all(sum(o.shape[0] for o in r.out) == r.rows.shape[0] for r in every)
    assert int(server.st.n_free) == n_pages and sorted(server.st.free.tolist()) == list(range(n_pages))
    assert server.st.len.tolist() == [0, 0, 0]


def test_a_request_that_does_not_fit_waits():
    cfg = LAYERS["dense_bf16"]
    gen = torch.Generator().manual_seed(1)
    server = PagedServer(cfg, {k: v.cuda() for k, v in make_weights(cfg, gen).items()}, 2, 4, 16, 32, max_len=64)
    big = Request(torch.randn((60, 512), generator=gen).bfloat16().cuda(), None)
    assert server.submit(big) and not server.submit(Request(big.rows[:1], None))       # all four pages are promised
    assert not server.submit(Request(torch.cat([big.rows, big.rows]), None))            # longer than max_len
    while server.step():
        pass
    assert server.submit(Request(big.rows[:1], None)) and big.out and sum(o.shape[0] for o in big.out) == 60
