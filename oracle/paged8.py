"""Plain definition of the paged cache in 8 bits: which pages a step gives to whom, what the pages hold after rows are written,
and what the rows of a step attend.

TEST INFRASTRUCTURE ONLY (see oracle/layer.py); shares no code with the HIP library.  One request, one page, one row after
the other; all arithmetic is float64.

Element (8 bits, E4M3 of the OCP 8-bit floating point format: S EEEE MMM, exponent bias 7):
    E = 0         : (-1)^S * M * 2^-9
    E = 1..15     : (-1)^S * (1 + M/8) * 2^(E - 7), except E = 15, M = 7: NaN; no infinities; the largest value is 448
Scale (8 bits, E8M0): 2^(e - 127), one per page and KV head for K and for V.  Of the values written to a page so far that
are finite, the largest in size is at most 448 scales, and e (>= 1) is the least for which that holds.  Finite sizes above TOP are
written as TOP, since the next value, 2^128, is none of bf16 or fp32."""
import numpy as np

from oracle.layer import gqa_attention


def e4m3_value(code):
    s, e, m = (code >> 7) & 1, (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return float("nan")
    v = m * 2.0 ** -9 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
    return -v if s else v


VALUES = np.array([e4m3_value(c) for c in range(256)])
TOP = 240.0 * 2.0 ** 120
_SIZES = VALUES[:127]      # the sizes there are, ascending


def to_e4m3(x):
    """Codes of the nearest values, ties to the even code; |x| <= 448 or NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_SIZES, a), 1, 126)
    lo = hi - 1
    up, down = _SIZES[hi] - a, a - _SIZES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(a >= 448.0, 126, code)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isnan(x), 127, code).astype(np.uint8)


def scale_byte(amax):
    e = 1
    while amax > 448.0 * 2.0 ** (e - 127):
        e += 1
    return e


def rope(x, rot):
    """x [R, H, hd], rot [R, hd / 2, 2] (cos, sin): rotate-half."""
    half = x.shape[-1] // 2
    c, s = rot[:, None, :, 0], rot[:, None, :, 1]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def plan(n_new, length, free, n_free, table, page_rows, max_rows):
    """One step.  Lists in, a dict of new lists out; `table` rows as wide as a request's pages may be many."""
    P, N = page_rows, len(n_new)
    pages = lambda rows: -(-rows // P)   # noqa: E731
    table, free, stack = [list(t) for t in table], list(free), list(free[:n_free])
    for i in range(N):
        if n_new[i] < 0:
            stack += table[i][:pages(length[i])]
    there, wanted = len(stack), 0
    out = dict(len=list(length), kv_len=[0] * N, cu=[0], slot=[-1] * max_rows, pos=[0] * max_rows, n_refused=0)
    for i in range(N):
        first = out["cu"][i]
        out["cu"].append(min(first + max(n_new[i], 0), 2 ** 31 - 1))
        if n_new[i] < 0:
            out["len"][i] = 0
        if n_new[i] <= 0:
            continue
        end = length[i] + n_new[i]
        for r in range(first, min(out["cu"][i + 1], max_rows)):
            out["pos"][r] = length[i] + r - first
        fits = end <= len(table[i]) * P and out["cu"][i + 1] <= max_rows
        need = pages(end) - pages(length[i])
        wanted += need if fits else 0
        if not fits or (need > 0 and wanted > there):
            out["n_refused"] += 1
            continue
        for c in range(pages(length[i]), pages(end)):
            table[i][c] = stack.pop()
        out["len"][i] = out["kv_len"][i] = end
        for r in range(first, out["cu"][i + 1]):
            p = out["pos"][r]
            out["slot"][r] = table[i][p // P] * P + p % P
    free[n_free:len(stack)] = stack[n_free:]
    return dict(out, table=table, free=free, n_free=len(stack))


class Pages:
    """Codes [page][row][head][hd] and scale bytes [page][head] of K and of V."""

    def __init__(self, n_pages, page_rows, n_heads, hd):
        self.P = page_rows
        self.codes = {n: np.zeros((n_pages, page_rows, n_heads, hd), np.uint8) for n in "kv"}
        self.scale = {n: np.ones((n_pages, n_heads), np.int64) for n in "kv"}

    def write(self, slots, k, v):
        """Rows k (rotated), v [R, heads, hd] to slots [R] (< 0: nowhere), as one call does: all rows of a page together."""
        bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))      # [R, heads]
        for page in sorted({int(s) // self.P for s in slots if s >= 0}):
            rows = [r for r, s in enumerate(slots) if s >= 0 and s // self.P == page]
            at = [int(slots[r]) % self.P for r in rows]
            held = min(at)                                             # rows written before
            for name, x in (("k", k), ("v", v)):
                for h in range(x.shape[1]):
                    y = x[rows, h]
                    amax = np.abs(np.where(np.isfinite(y), y, 0.0)).max()
                    old = self.scale[name][page, h]
                    new = scale_byte(amax) if held == 0 else max(scale_byte(amax), old)
                    self.scale[name][page, h] = new
                    c = self.codes[name][page, :, h]
                    if held and new > old:
                        c[:held] = to_e4m3(VALUES[c[:held]] * 2.0 ** float(old - new))
                    if name == "k":
                        y = np.where(bad[rows, h][:, None], np.nan, y)
                    else:
                        y = np.where(np.isfinite(y), y, 0.0)
                    c[at] = to_e4m3(np.clip(y, -TOP, TOP) / 2.0 ** float(new - 127))

    def rows(self, name, table_row, n):
        """The first n cached rows of a request, [n, heads, hd]."""
        pages = [table_row[c] for c in range(-(-n // self.P))]
        if not pages:
            return np.zeros((0,) + self.codes[name].shape[2:])
        x = VALUES[self.codes[name][pages]] * 2.0 ** (self.scale[name][pages].astype(np.float64) - 127)[:, None, :, None]
        return x.reshape((-1,) + x.shape[2:])[:n]


def attend(q, k, v):
    """q [n, Hq, hd]: the last n of the len(k) rows; row j sees rows 0 .. len(k) - n + j, and gives zeros where that is none."""
    n, out = q.shape[0], np.zeros(q.shape)
    sees = len(k) - n + np.arange(n) + 1
    some = sees > 0
    if some.any():
        out[some] = gqa_attention(q[some], k, v, sees[some])
    return out
