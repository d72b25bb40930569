"""Definition of the operators around 8-bit integer weights, in numpy float64: codes of rows, products of codes, the norms around a
block, routing by rules, the experts' products.  One row, one expert at a time; test infrastructure, shares no code with the library."""
import numpy as np


def row_codes(x):
    """x [rows, cols] of numbers that float32 holds -> (codes int64, scale float32).  127 x is exact in 64 bits, and its quotient by a 24-bit
    number is a tie only if it is one exactly."""
    x = np.asarray(x, dtype=np.float64)
    q, scale = np.zeros(x.shape, dtype=np.int64), np.zeros(len(x), dtype=np.float32)
    for i, row in enumerate(x):
        if not np.isfinite(row).all():
            scale[i] = np.nan
            continue
        amax = np.abs(row).max(initial=0.0)
        if amax > 0:
            q[i] = np.rint(127.0 * row / amax).astype(np.int64)
            scale[i] = np.float32(amax) / np.float32(127.0)
    return q, scale


def silu(z):
    with np.errstate(over="ignore"):
        return z / (1.0 + np.exp(-z))


def product(a, a_scale, b, b_scale):
    """a int [M, K], b int [N, K] -> float64 [M, N]"""
    s = np.asarray(a, dtype=np.int64) @ np.asarray(b, dtype=np.int64).T
    return s * np.asarray(a_scale, dtype=np.float64)[:, None] * np.asarray(b_scale, dtype=np.float64)


def rms_norm(x, g, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * g


def residual(x, b, g_post, gate, alpha, eps):
    if g_post is not None:
        b = rms_norm(b, g_post, eps)
    return x + alpha * (b if gate is None else gate * b)


def _gap(v, n):
    """v descending: the least distance, relative to the larger, of neighbours that differ, among the first n and up to the next smaller one."""
    gap = np.inf
    for i in range(len(v) - 1):
        if v[i] != v[i + 1] and v[i] < np.inf and v[i + 1] > -np.inf:
            gap = min(gap, (v[i] - v[i + 1]) / max(abs(v[i]), abs(v[i + 1])))
        if i >= n - 1 and v[i] != v[i + 1]:
            break
    return gap


def route(logits, bias, top_k, score, n_groups=1, topk_groups=1, group_top=1, renorm=True, factor=1.0):
    """One row after another; (idx, weight, gap): gap is the least distance, relative to the larger, of two
    different numbers that the choice or its order rests on."""
    E = logits.shape[1]
    S = E // n_groups
    idx, weight, gaps = [], [], []
    by_logit = bias is None and (topk_groups == n_groups or group_top == 1)    # scores are increasing functions of them
    for l in np.asarray(logits, dtype=np.float64):
        l = np.where(np.isnan(l), -np.inf, l)
        dead, top = l == -np.inf, l.max()
        with np.errstate(over="ignore", invalid="ignore"):
            if score == "sigmoid":
                s = np.where(dead, 0.0, 1.0 / (1.0 + np.exp(-l)))
            else:
                s = np.where(dead, 0.0, np.where(l == top, 1.0, np.exp(l - top)))
                s = s / s.sum() if s.sum() > 0 else s
            c = l if by_logit else s + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
        c = np.where(np.isnan(c) | dead, -np.inf, c)
        gap = np.inf
        ok = np.ones(E, dtype=bool)
        if topk_groups < n_groups:
            total = np.full(n_groups, -np.inf)
            for g in range(n_groups):
                live = sorted((v for v in c[g * S:(g + 1) * S] if v > -np.inf), reverse=True)[:group_top]
                if live:
                    total[g] = sum(live)
            order = sorted(range(n_groups), key=lambda g: (-total[g], g))
            gap = _gap(total[order], topk_groups)
            ok[:] = False
            for g in order[:topk_groups]:
                ok[g * S:(g + 1) * S] = True
        order = sorted((e for e in range(E) if ok[e]), key=lambda e: (-c[e], e))
        gap = min(gap, _gap(c[order], top_k))
        chosen = order[:top_k]
        w = s[chosen]
        if renorm:
            w = w / w.sum() if w.sum() > 0 else w
        idx.append(chosen)
        weight.append(w * factor)
        gaps.append(gap)
    return np.array(idx), np.array(weight), np.array(gaps)


def experts(m_q, m_scale, h, idx, weight, gate_up, gate_up_scale, down, down_scale, store):
    """y [rows, d]; store rounds an array to the storage type."""
    y = np.array(h, dtype=np.float64)
    F = gate_up.shape[1] // 2
    for t in range(len(y)):
        for e, w in zip(idx[t], weight[t]):
            if not 0 <= e < len(gate_up):
                continue
            gu = product(m_q[t:t + 1], m_scale[t:t + 1], gate_up[e], gate_up_scale[e])
            q, s = row_codes(store(silu(gu[:, :F]) * gu[:, F:]))
            y[t] += w * product(q, s, down[e], down_scale[e])[0]
    return y
