"""A continuous batch over the paged cache in 8 bits: requests arrive, prefill in chunks, decode and leave, and every step
runs whatever rows fit its budget -- the serving loop that the paper's server keeps around its layers (Sec. IV-B: chunked
prefill, one batch of prompt chunks and decode tokens).

    python -m paper_2605_23296_amd.paged_serving

One step is compact_paged_plan, then per layer RMSNorm, q/k/v projection, compact_rope_paged_write, compact_attn_paged, output
projection, and the feed-forward half.  The host knows how many rows each request brings; where they go is decided on the
GPU, and the host never reads it back.  Inputs of a request (prompt rows and the rows of its decode steps) are given, as
everywhere in this package: there is no output head.
"""
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


class PagedServer:
    """One layer (weights as for binding.Layer; dense or routed) that serves up to n_slots requests at a time from n_pages pages
    of page_rows rows, max_rows rows a step, max_len rows a request."""

    def __init__(self, layer, weights, n_slots, n_pages, page_rows, max_rows, max_len, device="cuda"):
        self.lay, self.cfg, self.device = B.Layer(layer, weights), layer, device
        self.slots, self.leaving, self.max_rows, self.max_len = [None] * n_slots, set(), max_rows, max_len
        self.kv = B.PagedKV.allocate(layer, n_slots, -(-max_len // page_rows), n_pages, page_rows, device)
        self.st = B.PagedStep(layer, n_slots, max_rows, device, n_pages=n_pages)
        need = max(self.lay.paged_workspace_bytes(n_slots, max_rows, max_rows, max_len), self.lay.workspace_bytes(max_rows, 64, 1))
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
        lay, c, w, dt = self.lay, self.cfg, self.lay.weights, x.dtype

        def empty(cols):
            return torch.empty((rows, cols), dtype=dt, device=self.device)
        n, qkv, q, o, h, m, y = (empty(k) for k in (c.d_model, c.Dq + 2 * c.Dkv, c.Dq, c.Dq, c.d_model, c.d_model, c.d_model))
        lay.compact_rmsnorm(x, w["g_attn"], n)
        lay.compact_gemm(n, w["w_qkv"], None, qkv)
        lay.compact_rope_paged_write(qkv, self.kv, self.st.slot, self.st.rot, q)
        lay.compact_attn_paged(q, self.kv, self.st.cu, self.st.kv_len, max_new, max(self.held), o)
        lay.compact_gemm(o, w["w_o"], x, h)
        lay.compact_rmsnorm(h, w["g_ffn"], m)
        if c.n_experts:
            idx = torch.empty((rows, c.top_k), dtype=torch.int32, device=self.device)
            gate = torch.empty((rows, c.top_k), dtype=torch.float32, device=self.device)
            lay.compact_moe_route(m, w["w_router"], idx, gate)
            lay.compact_moe_ffn(m, h, idx, gate, y)
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
    server = PagedServer(layer, make_weights(layer, gen, "cuda"), n_slots=24, n_pages=2048, page_rows=64, max_rows=2048, max_len=8192)

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
