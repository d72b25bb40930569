"""The serving loop from 8-bit integer weights, and under another routing rule: every row against the definition in 64 bits over the rows that the cache
holds; the bits of a request do not depend on its company."""
import numpy as np
import pytest
import torch

from oracle import int8 as I8
from oracle import layer as O
from oracle import paged8 as P8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.paged_serving import PagedServer, Request
from paper_2605_23296_amd.workloads import LayerConfig, make_weights, to_numpy_f64
from tests.util import BF16_VEC_TOL, vec_rel_err

pytestmark = pytest.mark.gpu

DENSE = LayerConfig(d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, ffn_dim=1024, rope_theta=500000.0, dtype="bf16")
LAYERS = {"dense_bf16": DENSE, "dense_fp32": LayerConfig(**dict(DENSE.as_dict(), d_model=256, n_q_heads=4, ffn_dim=512, dtype="fp32")),
          "routed_bf16": LayerConfig(**dict(DENSE.as_dict(), ffn_dim=320, n_experts=16, top_k=4))}
RULE = dict(score="sigmoid", n_groups=4, topk_groups=2, group_top=2, factor=1.5)


class Definition:
    """The layer from codes, in 64 bits; store rounds to the storage type where the layer stores rows."""

    def __init__(self, cfg, w):
        self.cfg, self.eps = cfg, cfg.rms_eps
        dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
        self.store = lambda x: torch.tensor(np.asarray(x)).to(dt).double().numpy()
        self.w = {k: to_numpy_f64(v) for k, v in w.items()}
        self.codes = {k: I8.row_codes(self.w[k].reshape(-1, self.w[k].shape[-1])) for k in self.w if k.startswith("w_") and k != "w_router"}
        self.ref = O.Layer(cfg.as_dict(), self.w)

    def linear(self, x, name):
        return I8.product(*I8.row_codes(x), *self.codes[name])

    def norm(self, x, name):
        return self.store(I8.rms_norm(x, self.w[name], self.eps))

    def qkv(self, x, pos):
        c = self.cfg
        n = self.norm(x, "g_attn")
        qkv = self.store(self.linear(n, "w_qkv")).reshape(len(x), -1, c.head_dim)
        q, k, v = qkv[:, :c.n_q_heads], qkv[:, c.n_q_heads:c.n_q_heads + c.n_kv_heads], qkv[:, c.n_q_heads + c.n_kv_heads:]
        half = c.head_dim // 2
        ang = np.asarray(pos, dtype=np.float64)[:, None] * c.rope_theta ** (-np.arange(half) / half)
        turn = np.exp(1j * ang)[:, None]
        rot = lambda t: np.concatenate([(z := (t[..., :half] + 1j * t[..., half:]) * turn).real, z.imag], -1)   # noqa: E731
        return rot(q), rot(k), v

    def rest(self, x, o, rule, bias, forced):
        """Rows behind the attention; forced: the experts that the router chose."""
        c = self.cfg
        h = self.store(x + self.store(self.linear(self.store(o), "w_o")))
        m = self.norm(h, "g_ffn")
        if not c.n_experts:
            gu = self.linear(m, "w_gate_up")
            return h + self.linear(self.store(I8.silu(gu[:, :c.ffn_dim]) * gu[:, c.ffn_dim:]), "w_down")
        s = 1 / (1 + np.exp(-m @ self.w["w_router"].T))
        c_all = s + bias
        if rule is not None:      # whoever was chosen is within the logits' noise of the definition's own choice
            own, _, _ = I8.route(m @ self.w["w_router"].T, bias, c.top_k, **rule)
            assert (np.take_along_axis(c_all, forced, -1).min(-1) > np.take_along_axis(c_all, own, -1).min(-1) - 0.02).all()
        w = np.take_along_axis(s, forced, -1)
        w = w / w.sum(-1, keepdims=True) * RULE["factor"]
        E, F, d = c.n_experts, c.ffn_dim, c.d_model
        (gu, gus), (dn, dns) = self.codes["w_exp_gate_up"], self.codes["w_exp_down"]
        return I8.experts(*I8.row_codes(m), h, forced, w, gu.reshape(E, 2 * F, d), gus.reshape(E, 2 * F), dn.reshape(E, d, F), dns.reshape(E, d), self.store)


@pytest.mark.parametrize("name", LAYERS)
def test_rows_of_a_continuous_batch_from_int8_weights(name, monkeypatch):
    cfg = LAYERS[name]
    gen = torch.Generator().manual_seed(7)
    w = make_weights(cfg, gen, gain_jitter=True)
    bias = 0.05 * torch.randn(16, generator=gen)
    definition = Definition(cfg, w)
    routed = cfg.n_experts > 0
    server = PagedServer(cfg, {k: v.cuda() for k, v in w.items()}, 3, 24, 16, 96, max_len=320, int8=True, route=B.RouteRule(**RULE) if routed else None,
                         route_bias=bias.cuda() if routed else None)
    chosen = []
    if routed:
        call = server.lay.compact_route

        def spy(rule, logits, b, idx, weight, **kw):
            call(rule, logits, b, idx, weight, **kw)
            chosen.append(idx)
        server.lay.compact_route = spy
    dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32

    def rows(n):
        return torch.randn((n, cfg.d_model), generator=gen).to(dt).cuda()
    waiting = [Request(rows(L), rows(S)) for L, S in ((150, 5), (1, 3), (17, 9), (64, 2))]
    compared = 0
    while True:
        while waiting and server.submit(waiting[0]):
            waiting.pop(0)
        before = [(r, None if r is None else r.done) for r in server.slots]
        if server.step() == 0 and not waiting:
            break
        at = 0
        for i, (r, d0) in enumerate(before):
            if r is None or r.done == d0:
                continue
            n = r.done - d0
            K, V = (to_numpy_f64(t) for t in server.kv.rows(i, r.done))
            x = to_numpy_f64(r.rows[d0:r.done])
            q, k, v = definition.qkv(x, np.arange(d0, r.done))
            o = P8.attend(definition.store(q), K, V).reshape(n, -1)
            y = definition.rest(x, o, RULE if routed else None, bias.double().numpy() if routed else 0.0, chosen[-1][at:at + n].cpu().numpy() if routed else None)
            # A row of codes whose values are off by e (a storage rounding, 2^-9 of them; 2^-20 with fp32) has some one code off: e / step of them by a
            # step, 1 / 127 of the largest: rms sqrt(e step), 0.5 % of the row with bf16, 0.02 % with fp32, four times on the way to y
            assert vec_rel_err(to_numpy_f64(r.out[-1]), y) < (BF16_VEC_TOL if cfg.dtype == "bf16" else 2e-3), (i, d0)
            # a cached code is within 2^-4 of its value, that within the projection's error of the head's size
            for cached, want in ((K[d0:], k), (V[d0:], v)):
                err = np.abs(cached - want)
                assert (err <= np.abs(want) * 2.0 ** -4 + np.abs(want).max() * 0.03).all()
            at += n
            compared += n
    assert compared == 150 + 5 + 1 + 3 + 17 + 9 + 64 + 2


@pytest.mark.parametrize("name", LAYERS)
def test_a_request_from_int8_weights_has_the_same_bits_alone(name):
    cfg = LAYERS[name]
    gen = torch.Generator().manual_seed(9)
    w = {k: v.cuda() for k, v in make_weights(cfg, gen, gain_jitter=True).items()}
    dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    data = [(torch.randn((L, cfg.d_model), generator=gen).to(dt).cuda(), torch.randn((6, cfg.d_model), generator=gen).to(dt).cuda()) for L in (30, 1, 64, 17)]

    def run(which):
        server = PagedServer(cfg, w, 4, 40, 16, 128, max_len=128, int8=True)
        rs = [Request(*data[i]) for i in which]
        assert all(server.submit(r) for r in rs)
        while server.step():
            pass
        return [torch.cat(r.out) for r in rs]
    together = run(range(4))
    for i in range(4):
        assert torch.equal(run([i])[0], together[i]), i


def test_another_routing_rule_in_the_serving_loop():
    """bf16 weights, the layer's own rule spelled out as a rule: the same rows."""
    cfg = LAYERS["routed_bf16"]
    gen = torch.Generator().manual_seed(3)
    w = {k: v.cuda() for k, v in make_weights(cfg, gen).items()}
    x = torch.randn((50, cfg.d_model), generator=gen).bfloat16().cuda()
    out = []
    for route in (None, B.RouteRule("softmax", renorm=True)):
        server = PagedServer(cfg, w, 1, 8, 16, 64, max_len=64, route=route)
        r = Request(x, None)
        assert server.submit(r)
        while server.step():
            pass
        out.append(torch.cat(r.out).double())
    # the weights of the experts differ by roundings of fp32: a row's elements by one step of bf16 here and there
    assert float((out[0] - out[1]).abs().max()) <= 2 * 2.0 ** -8 * float(out[0].abs().max())
