"""A continuous batch over the paged cache in 8 bits: requests arrive, prefill in chunks, decode and leave, and every step
runs whatever rows fit its budget -- the serving loop that the paper's server keeps around its layers (Sec. IV-B: chunked
prefill, one batch of prompt chunks and decode tokens).

    python -m paper_2605_23296_amd.paged_serving [--int8]

One step is compact_paged_plan, then per layer RMSNorm, q/k/v projection, compact_rope_paged_write, compact_attn_paged, output
projection, and the feed-forward half.  The host knows how many rows each request brings; where they go is decided on the
GPU, and the host never reads it back.  Inputs of a request (prompt rows and the rows of its decode steps) are given, as
everywhere in this package: there is no output head.

With int8=True the projections (and experts) run from 8-bit codes with a scale per output channel, and every projection's rows as codes with a scale per
row: compact_block_norm hands the normalised rows on as codes, compact_quant_i8 the attention's and the hidden ones.
"""
import sys

import torch

from . import binding as B


class Request:
    """prompt [L, d], decode [S, d]: the rows that the request feeds, in order; `out` collects the layer's rows for them."""

    def __init__(self, prompt, decode):
        self.rows = torch.cat([prompt, decode]) if decode is not None else prompt
        self.n_prompt, self.done, self.out = prompt.shape[0], 0, []

    def wants(self, budget):
        """Rows for the next step: a decode row, or as much of the prompt as fits."""
        left = self.rows.shape[0] - self.done
        return min(left, 1 if self.done >= self.n_prompt else min(budget, self.n_prompt - self.done))


def int8_weights(lay, weights):
    """The projections of `weights` as (codes, scales) under their names, experts as binding.ExpertsI8 under "experts"; the other tensors as they are."""
    out = dict(weights)

    def codes(name):
        w = out.pop(name)
        rows = w.reshape(-1, w.shape[-1])
        q, scale = torch.empty(rows.shape, dtype=torch.int8, device=w.device), torch.empty(rows.shape[0], dtype=torch.float32, device=w.device)
        lay.compact_quant_i8(rows, q, scale)
        return q.view(w.shape), scale.view(w.shape[:-1])
    for name in ("w_qkv", "w_o", "w_gate_up", "w_down"):
        if name in out:
            out[name] = codes(name)
    if "w_exp_gate_up" in out:
        out["experts"] = B.ExpertsI8(*codes("w_exp_gate_up"), *codes("w_exp_down"))
    return out


class PagedServer:
    """One layer (weights as for binding.Layer; dense or routed) that serves up to n_slots requests at a time from n_pages pages
    of page_rows rows, max_rows rows a step, max_len rows a request.  int8: the projections run from codes made of the weights.  route (routed
    layers): a binding.RouteRule in the place of the layer's own rule, route_bias fp32 [n_experts] its bias, or the own rule's."""

    def __init__(self, layer, weights, n_slots, n_pages, page_rows, max_rows, max_len, device="cuda", int8=False, route=None, route_bias=None):
        self.lay, self.cfg, self.device = B.Layer(layer, None if int8 else weights), layer, device
        self.route, self.route_bias, self.int8 = route, route_bias, int8
        self.w = int8_weights(self.lay, weights) if int8 else weights
        if layer.n_experts and route is None and (int8 or route_bias is not None):
            self.route = B.RouteRule()      # (the layer's own: softmax over the chosen logits)
        self.slots, self.leaving, self.max_rows, self.max_len = [None] * n_slots, set(), max_rows, max_len
        self.kv = B.PagedKV.allocate(layer, n_slots, -(-max_len // page_rows), n_pages, page_rows, device)
        self.st = B.PagedStep(layer, n_slots, max_rows, device, n_pages=n_pages)
        need = [self.lay.paged_workspace_bytes(n_slots, max_rows, max_rows, max_len)]
        if not int8:
            need.append(self.lay.workspace_bytes(max_rows, 64, 1))
        elif layer.n_experts:
            need.append(self.lay.moe_ffn_i8_workspace_bytes(max_rows))
        if int8:     # (only products of few rows use one)
            shapes = [(layer.Dq + 2 * layer.Dkv, layer.d_model, 0), (layer.d_model, layer.Dq, 0)]
            shapes += [] if layer.n_experts else [(layer.ffn_dim, layer.d_model, 1), (layer.d_model, layer.ffn_dim, 0)]
            need += [self.lay.gemm_i8_workspace_bytes(M, *shape) for shape in shapes for M in range(64, max_rows + 64, 64)]
        need = max(need)
        self.lay.ws = torch.empty(need, dtype=torch.uint8, device=device)
        self.held = [0] * n_slots      # rows cached, as the host expects them
        self.free = n_pages            # pages not promised to a request

    def submit(self, request):
        """Takes the request if there is a slot, and pages for all of its rows.  One without rows is done at once."""
        if request.rows.shape[0] == 0:
            return True
        pages = -(-request.rows.shape[0] // self.kv.page_rows)
        free = [i for i, r in enumerate(self.slots) if r is None and i not in self.leaving]
        if request.rows.shape[0] > self.max_len or not free or pages > self.free:
            return False
        self.slots[free[0]], self.free = request, self.free - pages
        return True

    def layer_rows(self, x, rows, max_new):
        """The layer over the packed rows x [rows, d] of a planned step."""
        lay, c, w, dt = self.lay, self.cfg, self.w, x.dtype

        def empty(cols, dt=dt):
            return torch.empty((rows, cols), dtype=dt, device=self.device)

        def routed(m):
            idx, gate = empty(c.top_k, torch.int32), empty(c.top_k, torch.float32)
            if self.route is None:
                lay.compact_moe_route(m, w["w_router"], idx, gate)
            else:
                lay.compact_route(self.route, empty(c.n_experts, torch.float32), self.route_bias, idx, gate, m=m, w_router=w["w_router"])
            return idx, gate

        def attention(qkv):
            q, o = empty(c.Dq), empty(c.Dq)
            lay.compact_rope_paged_write(qkv, self.kv, self.st.slot, self.st.rot, q)
            lay.compact_attn_paged(q, self.kv, self.st.cu, self.st.kv_len, max_new, max(self.held), o)
            return o
        qkv, h, m, y = (empty(k) for k in (c.Dq + 2 * c.Dkv, c.d_model, c.d_model, c.d_model))
        if self.int8:
            scale = torch.empty(rows, dtype=torch.float32, device=self.device)

            def codes(t):
                q = torch.empty(t.shape, dtype=torch.int8, device=self.device)
                lay.compact_quant_i8(t, q, scale)
                return q
            n = empty(c.d_model, torch.int8)
            lay.compact_block_norm(x, g_pre=w["g_attn"], q=n, q_scale=scale)
            lay.compact_gemm_i8(n, scale, *w["w_qkv"], None, qkv)
            o = attention(qkv)
            lay.compact_gemm_i8(codes(o), scale, *w["w_o"], None, y)
            lay.compact_block_norm(x, b=y, h=h, g_pre=w["g_ffn"], n=m if c.n_experts else None, q=n, q_scale=scale)
            if c.n_experts:
                lay.compact_moe_ffn_i8(w["experts"], n, scale, h, *routed(m), y)
            else:
                act = empty(c.ffn_dim)
                lay.compact_gemm_i8(n, scale, *w["w_gate_up"], None, act, epilogue=1)
                lay.compact_gemm_i8(codes(act), scale, *w["w_down"], h, y)
            return y
        n = empty(c.d_model)
        lay.compact_rmsnorm(x, w["g_attn"], n)
        lay.compact_gemm(n, w["w_qkv"], None, qkv)
        lay.compact_gemm(attention(qkv), w["w_o"], x, h)
        lay.compact_rmsnorm(h, w["g_ffn"], m)
        if c.n_experts:
            lay.compact_moe_ffn(m, h, *routed(m), y)
        else:
            act = empty(c.ffn_dim)
            lay.compact_gemm(m, w["w_gate_up"], None, act, epilogue=1)
            lay.compact_gemm(act, w["w_down"], h, y)
        return y

    def step(self):
        """One step over the requests that are there: decode rows first, the rest of the budget in prompt rows, in slot order.
        Returns the rows run."""
        n_new, budget = [0] * len(self.slots), self.max_rows
        for decoding in (True, False):
            for i, r in enumerate(self.slots):
                if r is not None and (r.done >= r.n_prompt) == decoding and budget:
                    n_new[i] = r.wants(budget)
                    budget -= n_new[i]
        for i in self.leaving:         # their pages go back before this step's rows take any
            n_new[i], self.held[i] = -1, 0
        self.leaving = set()
        rows = sum(max(n, 0) for n in n_new)
        if rows == 0 and -1 not in n_new:
            return 0
        self.st.n_new.copy_(torch.tensor(n_new, dtype=torch.int32))
        self.lay.compact_paged_plan(self.kv, self.st)
        if rows:
            self.held = [h + max(n, 0) for h, n in zip(self.held, n_new)]
            x = torch.cat([r.rows[r.done:r.done + n] for r, n in zip(self.slots, n_new) if n > 0])
            # the plan's arrays hold max_rows rows; those behind the step's own are nobody's
            y = self.layer_rows(x.contiguous(), rows, max(n_new))
            at = 0
            for i, n in enumerate(n_new):
                if n <= 0:
                    continue
                r = self.slots[i]
                r.out.append(y[at:at + n])
                r.done += n
                at += n
                if r.done == r.rows.shape[0]:
                    self.slots[i] = None
                    self.leaving.add(i)
                    self.free += -(-r.done // self.kv.page_rows)
        self.st.advance()
        return rows


def main():
    from .workloads import DENSE_8B, LayerConfig, make_weights
    layer = LayerConfig(**DENSE_8B)
    gen = torch.Generator(device="cuda").manual_seed(0)
    server = PagedServer(layer, make_weights(layer, gen, "cuda"), n_slots=24, n_pages=2048, page_rows=64, max_rows=2048, max_len=8192,
                         int8="--int8" in sys.argv[1:])

    def rows(n):
        return torch.randn((n, layer.d_model), generator=gen, device="cuda").bfloat16()
    waiting = [Request(rows(200 + 331 * k % 4000), rows(32 + 7 * k % 64)) for k in range(48)]
    total = sum(r.rows.shape[0] for r in waiting)
    torch.cuda.synchronize()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    steps = done = 0
    while True:
        while waiting and server.submit(waiting[0]):
            waiting.pop(0)
        ran = server.step()
        if ran == 0 and not waiting:
            break
        done, steps = done + ran, steps + 1
    end.record()
    torch.cuda.synchronize()
    assert done == total
    ms = start.elapsed_time(end)
    print("48 requests, %d rows in %d steps: %.1f ms, %.0f k rows/s per layer" % (total, steps, ms, total / ms))
    print("pages free at the end: %d of %d" % (int(server.st.n_free), server.kv.n_pages))


if __name__ == "__main__":
    main()
