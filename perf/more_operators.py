"""The operators of a layer that is served from 8-bit integer weights, as cases that can be timed and checked: the norms around a
block with its gate, its residual and the codes of the rows that leave, the quantisation of rows, the product of two matrices
of codes, routing by scores with a bias and groups, and the routed experts' products.

A case is a dict of plain values; `op` is norm, quant, gemm, route or moe.

Codes: a row of values x with amax = max |x| is held as q = round(127 x / amax), ties to even, in -127 .. 127, and the scale amax / 127
in 32 bits.  Rows of activations and rows of a weight matrix [out, in] (its output channels) are quantised alike, so that a
product is C[m, n] = scale_a[m] scale_b[n] sum_k a[m, k] b[n, k].

Norm: with a block's output b, h = x + alpha * gate * RMSNorm(b; g_post), n = RMSNorm(h; g_pre); h and n are rounded to the storage type
where they are stored, the codes are those of n.

Routing: s = softmax or sigmoid of a row's logits, c = s + bias.  The experts lie in groups of neighbours; a group counts as the sum of
its `group_top` largest c, and only experts of the `topk_groups` best groups are eligible.  The top_k largest c among these are chosen, in that
order, and weigh s * factor, divided before by the sum of the chosen s where `renorm` says so.  Ties go to the lowest index.

Experts: y = h + sum_j w_j Down_j(codes(silu(Gate_j m) * Up_j m)); the rows between the products are held in the storage type and then as codes."""
import math
import random

import torch

own = False   # False: the plain forms below; True: the framework's operators

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # a decode step of 8 workers: both norms, a learned gate per channel, codes for the next projection
        dict(name="norm_decode_8", op="norm", dtype="bf16", rows=8, d=4096, post=True, gate="vector", alpha=1.0, out="codes"),
        # the headline prefill's rows between attention and feed-forward half
        dict(name="norm_8x4096", op="norm", dtype="bf16", rows=32768, d=4096, post=False, gate="none", alpha=1.0, out="rows"),
        # the attention output of 24 workers before its projection
        dict(name="quant_24", op="quant", dtype="bf16", rows=24, cols=4096),
        # the hidden rows of a chunk of prompts, an odd number of them
        dict(name="quant_1652", op="quant", dtype="bf16", rows=1652, cols=14336),
        # gate and up projection of a decode step of 8 workers
        dict(name="gemm_decode_8", op="gemm", dtype="bf16", M=8, N=14336, K=4096, glu=True, res=False),
        # down projection of a decode step of 64 workers
        dict(name="gemm_decode_64", op="gemm", dtype="bf16", M=64, N=4096, K=14336, glu=False, res=True),
        # an odd chunk of prompts through the routed layer's q/k/v projection
        dict(name="gemm_1001", op="gemm", dtype="bf16", M=1001, N=5120, K=2880, glu=False, res=False),
        # gate and up projection of the headline prefill
        dict(name="gemm_8x4096", op="gemm", dtype="bf16", M=32768, N=14336, K=4096, glu=True, res=False),
        # routing of 64 decode rows, softmax scores
        dict(name="route_decode_64", op="route", rows=64, E=128, top_k=4, score="softmax", bias=False, groups=1, topk_groups=1, group_top=1, renorm=True),
        # routing of 16 blocks of 8 k: sigmoid scores, a balancing bias, 8 groups
        dict(name="route_16x8192", op="route", rows=131072, E=256, top_k=8, score="sigmoid", bias=True, groups=8, topk_groups=4, group_top=2, renorm=True),
        # the routed layer's experts in a decode step of 16 workers
        dict(name="moe_decode_16", op="moe", rows=16, d=2880, F=2880, E=128, top_k=4),
        # and in a chunk of 16 k prompt rows
        dict(name="moe_16384", op="moe", rows=16384, d=2880, F=2880, E=128, top_k=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "quant", "gemm", "gemm", "gemm", "gemm", "route", "route", "moe", "moe"])
    dt = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "norm":
        d = rng.choice([64, 256, 512, 1088, 2048, 2880, 4096, 4096, 8192])
        return dict(op=op, dtype=dt, rows=_log(rng, 1, min(65536, 32768 * 2048 // d)), d=d, post=rng.random() < 0.5,
                    gate=rng.choice(["none", "vector", "rows"]), alpha=rng.choice([1.0, 0.5, 0.22]), out=rng.choice(["codes", "rows"]))
    if op == "quant":
        cols = rng.choice([64, 200, 1000, 2880, 4096, 6144, 14336, 28672])
        return dict(op=op, dtype=dt, rows=_log(rng, 1, min(65536, 32768 * 4096 // cols)), cols=cols)
    if op == "gemm":
        N, K = rng.choice([(6144, 4096), (4096, 4096), (14336, 4096), (4096, 14336), (5120, 2880), (2880, 4096), (2880, 2880), (512, 256),
                           (1024, 256), (256, 1024), (rng.randint(1, 5000), 16 * rng.randint(1, 500))])
        glu = rng.random() < 0.35
        return dict(op=op, dtype=dt, M=_log(rng, 1, rng.choice([16, 64, 1024, 16384])), N=N, K=K, glu=glu, res=not glu and rng.random() < 0.5)
    if op == "route":
        E = rng.choice([8, 16, 64, 128, 160, 256, 256])
        groups = rng.choice([1, 1, 4, 8]) if E > 8 else rng.choice([1, 2])
        tg = rng.randint(1, groups)
        return dict(op=op, rows=_log(rng, 1, 131072), E=E, top_k=rng.randint(1, min(8, tg * (E // groups))), score=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.6, groups=groups, topk_groups=tg, group_top=rng.choice([1, 2]), renorm=rng.random() < 0.7)
    d, F, E = rng.choice([(2880, 2880, 128), (2880, 2880, 32), (1024, 1408, 64), (512, 192, 16), (4096, 1408, 8)])
    return dict(op=op, rows=_log(rng, 1, 8192), d=d, F=F, E=E, top_k=rng.randint(1, min(8, E)))


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _rows(shape, gen):
    """Activations: a few strong channels, rows of different size."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x[..., 5::61] *= 6.0
    return x.mul_(torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda")))


def _codes(x):
    """(codes, scales) of the rows of x, as a program has them from the quantising operator."""
    amax = x.abs().amax(-1, keepdim=True)
    return torch.round(x * (127.0 / amax)).clamp_(-127, 127).to(torch.int8), (amax / 127.0).squeeze(-1)


def _weight_codes(shape, gen, size):
    """Codes and scales of weights N(0, size): a row's largest of some thousand lies near 4 of them."""
    q = (torch.randn(shape, generator=gen, device="cuda") * 31.0).round_().clamp_(-127, 127).to(torch.int8)
    s = size / 31.0 * (1.0 + 0.1 * torch.rand(shape[:-1], generator=gen, device="cuda"))
    return q, s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], dict(case=case)
    dt = DTYPES[case.get("dtype", "bf16")]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    if op == "norm":
        n, d = case["rows"], case["d"]
        s.update(x=_rows((n, d), gen).to(dt), b=_rows((n, d), gen).to(dt), g_post=(1 + 0.1 * normal(d)).to(dt) if case["post"] else None,
                 g_pre=(1 + 0.1 * normal(d)).to(dt), gate=None, h=torch.empty((n, d), dtype=dt, device="cuda"))
        if case["gate"] != "none":
            s["gate"] = (0.5 + 0.3 * (normal(d) if case["gate"] == "vector" else normal(n, d))).to(dt)
    elif op == "quant":
        n, d = case["rows"], case["cols"]
        s["x"] = _rows((n, d), gen).to(dt)
    elif op == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"], s["a_scale"] = _codes(_rows((M, K), gen))
        s["b"], s["b_scale"] = _weight_codes(((2 if case["glu"] else 1) * N, K), gen, 1.0 / math.sqrt(K))
        s["r"] = normal(M, N).to(dt) if case["res"] else None
        s["c"] = torch.empty((M, N), dtype=dt, device="cuda")
    elif op == "route":
        n, E = case["rows"], case["E"]
        # some experts are liked more than others; the bias works against that
        liked = normal(E)
        s["logits"] = 1.5 * normal(n, E) + 0.7 * liked
        s["bias"] = (-0.05 * liked + 0.02 * normal(E)) if case["bias"] else None
        s["idx"] = torch.empty((n, case["top_k"]), dtype=torch.int32, device="cuda")
        s["w"] = torch.empty((n, case["top_k"]), dtype=torch.float32, device="cuda")
    else:
        n, d, F, E, k = (case[c] for c in ("rows", "d", "F", "E", "top_k"))
        s["m"], s["m_scale"] = _codes(_rows((n, d), gen))
        s["h"] = normal(n, d).bfloat16()
        s["gate_up"], s["gate_up_scale"] = _weight_codes((E, 2 * F, d), gen, 1.0 / math.sqrt(d))
        s["down"], s["down_scale"] = _weight_codes((E, d, F), gen, 1.0 / math.sqrt(F))
        score = normal(n, E) + 0.5 * normal(E)      # uneven loads
        top = torch.topk(score, k, dim=-1)
        s["idx"], s["w"] = top.indices.int(), torch.softmax(top.values, -1)
        s["y"] = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    if op in ("norm", "quant"):
        # what leaves: rows, or codes and scales (and room for the values that they stand for)
        s["n"] = torch.empty((n, d), dtype=dt, device="cuda")
        s["q"] = torch.empty((n, d), dtype=torch.int8, device="cuda")
        s["q_scale"] = torch.empty(n, dtype=torch.float32, device="cuda")
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _plain_codes(x):
    """Codes (as 32-bit numbers) and scales of the rows of x; the quotient in 64 bits: half codes are common, at x = amax / 2."""
    amax = x.float().abs().amax(-1, keepdim=True)
    return torch.round(x.double() * 127.0 / amax.double()).float(), amax / 127.0


def _rms(x, g):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * g.float()


def _plain_norm(s):
    dt, b = s["x"].dtype, s["b"].float()
    if s["g_post"] is not None:
        b = _rms(b, s["g_post"])
    if s["gate"] is not None:
        b = b * s["gate"].float()
    h = (s["x"].float() + s["case"]["alpha"] * b).to(dt)
    n = _rms(h.float(), s["g_pre"]).to(dt)
    if s["case"]["out"] == "codes":
        q, scale = _plain_codes(n)
        n = (q * scale).to(dt)
    return dict(h=h, n=n)


def _plain_quant(s):
    q, scale = _plain_codes(s["x"])
    return dict(x=(q * scale).to(s["x"].dtype), scale=scale.squeeze(-1))


def _plain_gemm(s):
    c = (s["a"].float() @ s["b"].float().t()) * s["a_scale"][:, None] * s["b_scale"]
    if s["case"]["glu"]:
        g, u = c.chunk(2, -1)
        c = g / (1.0 + torch.exp(-g)) * u
    if s["r"] is not None:
        c = c + s["r"].float()
    return c.to(s["c"].dtype)


def _descending(x):
    return torch.sort(x, dim=-1, descending=True, stable=True)


def _plain_route(s):
    c, x = s["case"], s["logits"].double()      # (in 64 bits: 131072 rows hold borders that 32 bits do not tell apart)
    if c["score"] == "sigmoid":
        p = 1.0 / (1.0 + torch.exp(-x))
    else:
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
    v = p if s["bias"] is None else p + s["bias"].double()
    if c["groups"] > 1:
        grouped = v.view(c["rows"], c["groups"], -1)
        best = _descending(_descending(grouped)[0][..., :c["group_top"]].sum(-1))[1][:, :c["topk_groups"]]
        live = torch.zeros(grouped.shape[:2], dtype=torch.bool, device=v.device).scatter_(1, best, True)
        v = torch.where(live[..., None], grouped, -math.inf).view(v.shape)
    idx = _descending(v)[1][:, :c["top_k"]].contiguous()
    w = p.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    return dict(idx=idx.int(), w=w.float())


def _plain_moe(s):
    c = s["case"]
    n, k, E = c["rows"], c["top_k"], c["E"]
    flat = s["idx"].long().view(-1)
    # only experts that have rows; the rows of each side by side, padded to the most
    used, at = torch.unique(flat, return_inverse=True)
    order = torch.argsort(at, stable=True)
    count = torch.bincount(at)
    place = torch.arange(n * k, device=flat.device) - (count.cumsum(0) - count)[at[order]]
    cap = int(count.max())

    def products(rows, scale, w, w_scale):
        """rows [n k, K] of codes in the order of experts -> [n k, N]"""
        x = torch.zeros((used.numel(), cap, rows.shape[1]), device=rows.device)
        x[at[order], place] = rows
        out = torch.matmul(w[used].float(), x.transpose(1, 2).contiguous()).transpose(1, 2)[at[order], place]
        return out * scale * w_scale[used][at[order]]
    g, u = products(s["m"].float()[order // k], s["m_scale"][order // k, None], s["gate_up"], s["gate_up_scale"]).chunk(2, -1)
    q, scale = _plain_codes((g / (1.0 + torch.exp(-g)) * u).bfloat16())
    out = products(q, scale, s["down"], s["down_scale"]) * s["w"].view(-1)[order, None]
    back = torch.empty_like(out)
    back[order] = out
    return (s["h"].float() + back.view(n, k, -1).sum(1)).bfloat16()


# ---- the framework's operators -------------------------------------------------------------------------------------------

_handles = {}


def _layer(dtype="bf16", d=4096, F=64, E=0, k=0):
    """The layer handle that a program keeps."""
    from paper_2605_23296_amd import binding as B
    from paper_2605_23296_amd.workloads import LayerConfig
    key = (dtype, d, F, E, k)
    if key not in _handles:
        _handles[key] = B.Layer(LayerConfig(d_model=d, n_q_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=F, n_experts=E, top_k=k, rms_eps=EPS, dtype=dtype), None)
    return B, _handles[key]


def _values(s):
    return torch.mul(s["q"], s["q_scale"][:, None], out=s["n"])


def _own_norm(s):
    lay = _layer(s["case"]["dtype"], s["case"]["d"])[1]
    codes = s["case"]["out"] == "codes"
    lay.compact_block_norm(s["x"], b=s["b"], g_post=s["g_post"], gate=s["gate"], alpha=s["case"]["alpha"], h=s["h"], g_pre=s["g_pre"],
                           n=None if codes else s["n"], q=s["q"] if codes else None, q_scale=s["q_scale"] if codes else None)
    return dict(h=s["h"], n=_values(s) if codes else s["n"])


def _own_quant(s):
    _layer(s["case"]["dtype"])[1].compact_quant_i8(s["x"], s["q"], s["q_scale"])
    return dict(x=_values(s), scale=s["q_scale"])


def _own_gemm(s):
    c, lay = s["case"], _layer(s["case"]["dtype"])[1]
    if "ws" not in s:
        s["ws"] = torch.empty(lay.gemm_i8_workspace_bytes(c["M"], c["N"], c["K"], int(c["glu"])), dtype=torch.uint8, device="cuda")
    lay.ws = s["ws"]
    lay.compact_gemm_i8(s["a"], s["a_scale"], s["b"], s["b_scale"], s["r"], s["c"], epilogue=int(c["glu"]))
    return s["c"]


def _own_route(s):
    c = s["case"]
    B, lay = _layer(E=c["E"], k=c["top_k"])
    if "rule" not in s:
        s["rule"] = B.RouteRule(score=c["score"], n_groups=c["groups"], topk_groups=c["topk_groups"], group_top=c["group_top"], renorm=c["renorm"])
    lay.compact_route(s["rule"], s["logits"], s["bias"], s["idx"], s["w"])
    return dict(idx=s["idx"], w=s["w"])


def _own_moe(s):
    c = s["case"]
    B, lay = _layer(d=c["d"], F=c["F"], E=c["E"], k=c["top_k"])
    if "experts" not in s:
        s["experts"] = B.ExpertsI8(s["gate_up"], s["gate_up_scale"], s["down"], s["down_scale"])
        s["ws"] = torch.empty(lay.moe_ffn_i8_workspace_bytes(c["rows"]), dtype=torch.uint8, device="cuda")
    lay.ws = s["ws"]
    lay.compact_moe_ffn_i8(s["experts"], s["m"], s["m_scale"], s["h"], s["idx"], s["w"], s["y"])
    return s["y"]


def run(state):
    if own:
        return {"norm": _own_norm, "quant": _own_quant, "gemm": _own_gemm, "route": _own_route, "moe": _own_moe}[state["case"]["op"]](state)
    return {"norm": _plain_norm, "quant": _plain_quant, "gemm": _plain_gemm, "route": _plain_route, "moe": _plain_moe}[state["case"]["op"]](state)


def work(case):
    op, es = case["op"], 4 if case.get("dtype") == "fp32" else 2
    if op == "norm":
        n, d = case["rows"], case["d"]
        gate = {"none": 0, "vector": d, "rows": n * d}[case["gate"]]
        left = n * d + 4 * n if case["out"] == "codes" else es * n * d
        return dict(bytes=es * (3 * n * d + gate + (2 if case["post"] else 1) * d) + left, flops=(12 + (4 if case["post"] else 0)) * n * d)
    if op == "quant":
        return dict(bytes=(es + 1) * case["rows"] * case["cols"] + 4 * case["rows"], flops=3 * case["rows"] * case["cols"])
    if op == "gemm":
        M, N, K, f = case["M"], case["N"], case["K"], 2 if case["glu"] else 1
        return dict(bytes=M * K + f * N * K + 4 * (M + f * N) + es * M * N * (2 if case["res"] else 1), flops=2 * M * N * K * f)
    if op == "route":
        return dict(bytes=4 * case["rows"] * case["E"] + 8 * case["rows"] * case["top_k"], flops=25 * case["rows"] * case["E"])
    n, d, F, E, k = (case[c] for c in ("rows", "d", "F", "E", "top_k"))
    hit = E * (1 - (1 - k / E) ** n)      # experts that evenly spread rows reach
    return dict(bytes=int(hit * (3 * F * d + 4 * (2 * F + d))) + n * (5 * d + 4 + 8 * k), flops=6 * n * k * d * F)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def _code_values(x):
    """What the codes of the rows of x stand for: the multiples of amax / 127 next to its values."""
    step = x.abs().max(dim=-1, keepdim=True).values / 127.0
    return torch.round(x / step) * step


def _stored(x, dtype):
    return x.to(dtype).double()


def _unit(x):
    return x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS)


def _exact_norm(s):
    dt, branch = s["x"].dtype, s["b"].double()
    if s["g_post"] is not None:
        branch = _unit(branch).mul_(s["g_post"].double())
    if s["gate"] is not None:
        branch = branch.mul_(s["gate"].double())
    h = torch.add(s["x"].double(), branch, alpha=s["case"]["alpha"])
    n = _unit(_stored(h, dt)) * s["g_pre"].double()
    return dict(h=h, n=_code_values(_stored(n, dt)) if s["case"]["out"] == "codes" else n)


def _exact_quant(s):
    x = s["x"].double()
    return dict(x=_code_values(x), scale=x.abs().max(-1).values / 127.0)


def _silu_mul(g, u):
    return u * g * torch.sigmoid(g)


def _exact_gemm(s):
    N, out = s["case"]["N"], []
    b = s["b"].double() * s["b_scale"].double()[:, None]
    for lo in range(0, s["case"]["M"], 8192):
        a = s["a"][lo:lo + 8192].double() * s["a_scale"][lo:lo + 8192].double()[:, None]
        c = torch.mm(a, b.t())
        if s["case"]["glu"]:
            c = _silu_mul(c[:, :N], c[:, N:])
        out.append(c if s["r"] is None else c + s["r"][lo:lo + 8192].double())
    return torch.cat(out)


def _exact_route(s):
    """Every chosen expert by counting the experts before it."""
    c, x = s["case"], s["logits"].double()
    E, k, S = c["E"], c["top_k"], c["E"] // c["groups"]
    n = torch.arange(E, device=x.device)
    idx, w = [], []
    for lo in range(0, c["rows"], 4096):
        p = torch.sigmoid(x[lo:lo + 4096]) if c["score"] == "sigmoid" else torch.softmax(x[lo:lo + 4096], -1)
        v = p if s["bias"] is None else p + s["bias"].double()
        if c["groups"] > 1:
            total = v.unflatten(-1, (c["groups"], S)).topk(min(c["group_top"], S), -1).values.sum(-1)
            j = torch.arange(c["groups"], device=x.device)
            before = ((total[:, None, :] > total[:, :, None]) | ((total[:, None, :] == total[:, :, None]) & (j < j[:, None]))).sum(-1)
            v = v.masked_fill((before >= c["topk_groups"]).repeat_interleave(S, -1), -math.inf)
        rank = ((v[:, None, :] > v[:, :, None]) | ((v[:, None, :] == v[:, :, None]) & (n < n[:, None]))).sum(-1)
        chosen = torch.argsort(rank, -1)[:, :k]
        ws = p.gather(1, chosen)
        idx.append(chosen.int())
        w.append(ws / ws.sum(-1, keepdim=True) if c["renorm"] else ws)
    return dict(idx=torch.cat(idx), w=torch.cat(w))


def _exact_moe(s):
    m = s["m"].double() * s["m_scale"].double()[:, None]
    y, F = s["h"].double(), s["case"]["F"]
    for e in range(s["case"]["E"]):
        row, j = torch.nonzero(s["idx"] == e, as_tuple=True)
        if not row.numel():
            continue
        gu = torch.mm(m[row], (s["gate_up"][e].double() * s["gate_up_scale"][e].double()[:, None]).t())
        act = _code_values(_stored(_silu_mul(gu[:, :F], gu[:, F:]), torch.bfloat16))
        out = torch.mm(act, (s["down"][e].double() * s["down_scale"][e].double()[:, None]).t())
        y.index_add_(0, row, out * s["w"][row, j].double()[:, None])
    return y


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "quant": _exact_quant, "gemm": _exact_gemm, "route": _exact_route, "moe": _exact_moe}[case["op"]](s)
