"""Paged cache in 8 bits on the GPU against its plain definition in 64 bits (oracle/paged8.py): the plan of a step, the
write of new rows, the attention over the pages, and the three as a serving loop calls them."""
import numpy as np
import pytest
import torch

from oracle import paged8 as P8
from paper_2605_23296_amd import binding as B
from paper_2605_23296_amd.workloads import LayerConfig

pytestmark = pytest.mark.gpu
DEV = "cuda"


def layer(hq, hkv, hd, dtype="bf16", theta=10000.0):
    return LayerConfig(d_model=64 * hq, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, ffn_dim=256, rope_theta=theta, dtype=dtype)


def handle(lc):
    return B.Layer(lc, None)


def tdtype(lc):
    return torch.bfloat16 if lc.dtype == "bf16" else torch.float32


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


# ---- plan ----------------------------------------------------------------------------------------------------------------

def plan_both(lc, P, width, n_pages, n_new, length, max_rows, seed=0, room=None):
    """One step on the GPU and by definition; returns the GPU's step and table."""
    rng = np.random.default_rng(seed)
    perm = rng.permutation(n_pages).tolist()
    table, at = [], 0
    for L in length:
        n = -(-L // P)
        table.append(perm[at:at + n] + [-7] * (width - n))
        at += n
    assert at <= n_pages
    free = perm[at:] + [-9] * at
    n_free = n_pages - at if room is None else min(room, n_pages - at)
    want = P8.plan(n_new, length, free, n_free, table, P, max_rows)
    lay, t = handle(lc), ints(table)
    empty = torch.empty(0, dtype=torch.uint8, device=DEV)
    kv = B.PagedKV(lc, empty, empty, empty, empty, t, n_pages=n_pages, page_rows=P)
    st = B.PagedStep(lc, len(n_new), max_rows, DEV, n_new=ints(n_new), len=ints(length), free=ints(free), n_free=ints([n_free]))
    lay.compact_paged_plan(kv, st)
    for name, got, ref in (("cu", st.cu, want["cu"]), ("len", st.len_out, want["len"]), ("kv_len", st.kv_len, want["kv_len"]),
                           ("n_free", st.n_free_out, [want["n_free"]]), ("n_refused", st.n_refused, [want["n_refused"]]),
                           ("table", t, want["table"]), ("free", st.free, want["free"]), ("slot", st.slot, want["slot"])):
        assert got.tolist() == ref, name
    ang = np.array(want["pos"], dtype=np.float64)[:, None] * lc.rope_theta ** (-np.arange(lc.head_dim // 2) / (lc.head_dim // 2))
    # cos and sin rounded once to fp32; the angle carries a few units of 2^-53 of itself
    bound = 2.0 ** -24 + ang.max() * 2.0 ** -48
    assert np.abs(f64(st.rot) - np.stack([np.cos(ang), np.sin(ang)], -1)).max() <= bound
    return st, want


@pytest.mark.parametrize("n", [1, 2, 63, 255, 256, 257, 700, 4096])
def test_plan_of_decode_steps(n):
    rng = np.random.default_rng(n)
    length = rng.integers(0, 70, n).tolist()
    _, want = plan_both(layer(4, 2, 64), 16, 6, 6 * n + 1, [1] * n, length, n + 5, seed=n)
    assert want["n_refused"] == 0


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_plan_of_busy_steps(P, hd, seed):
    """Requests that decode, rest, have finished, arrive and go on with their prompts; few pages are free in two of three."""
    rng = np.random.default_rng(100 * P + seed)
    n = int(rng.integers(3, 400))
    kind = rng.integers(0, 5, n)
    n_new = np.choose(kind, [np.ones(n, int), np.zeros(n, int), -rng.integers(1, 9, n), rng.integers(1, 300, n), rng.integers(1, 65, n)]).tolist()
    length = np.where(kind == 3, 0, rng.integers(0, 5 * P, n)).tolist()
    width = 5 + (-(-300 // P))
    held = sum(-(-v // P) for v in length)
    lacks = sum(-(-(a + max(b, 0)) // P) - -(-a // P) for a, b in zip(length, n_new))
    n_pages = held + [lacks + 2, lacks // 2, 1][seed]
    st, want = plan_both(layer(4, 2, hd, theta=500000.0), P, width, n_pages, n_new, length, sum(max(v, 0) for v in n_new) + 3, seed=seed)
    assert seed > 0 or want["n_refused"] == 0


def test_plan_refuses_what_does_not_fit():
    lc = layer(4, 2, 64)
    # beyond the table's width (33 rows in pages of 16, two of them), beyond max_rows (the third), one that fits behind them
    _, want = plan_both(lc, 16, 2, 20, [33, 32, 40, 1], [0, 0, 0, 31], 70)
    assert want["kv_len"] == [0, 32, 0, 0] and want["n_refused"] == 3
    _, want = plan_both(lc, 16, 2, 20, [1, 32, 1], [32, 0, 31], 40)
    assert want["kv_len"] == [0, 32, 32] and want["n_refused"] == 1
    # no page left at all: rows that stay inside a page go on
    _, want = plan_both(lc, 16, 4, 4, [1, 1, 1], [16, 17, 1], 8, room=0)
    assert want["kv_len"] == [0, 18, 2]
    # nothing to do
    _, want = plan_both(lc, 16, 4, 4, [0, 0], [16, 0], 8)
    assert want["cu"] == [0, 0, 0] and want["kv_len"] == [0, 0]
    # the pages given back are all there are, and are taken in the same step
    _, want = plan_both(lc, 16, 4, 4, [-1, 64], [64, 0], 64, room=0)
    assert want["kv_len"] == [0, 64] and want["n_free"] == 0
    # sums beyond 31 bits do not wrap around
    _, want = plan_both(lc, 16, 4, 8, [2 ** 31 - 1, 3, 1], [0, 0, 5], 8)
    assert want["kv_len"] == [0, 0, 0]


# ---- write ---------------------------------------------------------------------------------------------------------------

def gpu_pages(lc, n_pages, P, table, fill):
    kv = B.PagedKV.allocate(lc, len(table), len(table[0]), n_pages, P, DEV)
    for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
        t.fill_(fill)
    kv.table.copy_(ints(table))
    return kv


def compare_pages(kv, ref, live):
    """Codes and scales of the rows that are live, bit for bit; live: {page: rows}."""
    for page, n in live.items():
        k, v = kv.k[page].cpu().numpy(), kv.v[page].cpu().numpy()
        want_k, want_v = ref.codes["k"][page, :n].transpose(1, 0, 2), ref.codes["v"][page, :n].transpose(1, 2, 0)
        got_k = np.where(k[:, :n] & 127 == 127, 127, k[:, :n])          # (a NaN has two codes)
        assert np.array_equal(kv.k_scale[page].cpu().numpy(), ref.scale["k"][page]), page
        assert np.array_equal(kv.v_scale[page].cpu().numpy(), ref.scale["v"][page]), page
        assert np.array_equal(got_k, want_k), page
        assert np.array_equal(v[:, :, :n], want_v), page


WRITE_LAYERS = [layer(4, 1, 64), layer(8, 2, 128), layer(10, 2, 64), layer(4, 2, 64, "fp32"), layer(3, 3, 128, "fp32")]


@pytest.mark.parametrize("lc", WRITE_LAYERS, ids=lambda c: "%d_%d_%d_%s" % (c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype))
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("steps", [[[1, 15, 16, 17], [1, 1, 1, 1], [200, 0, 47, 130], [1, 1, 1, 1]], [[300, 1, 5, 64], [1, 30, 0, 64]]])
def test_written_pages_hold_the_rounded_rows(lc, P, steps):
    """Rows whose rotation is by nothing: scales and codes bit for bit, over several calls whose values grow and shrink (so
    that pages are rounded again), into pages full of an earlier tenant's NaN."""
    rng = np.random.default_rng(P + lc.head_dim)
    N, Hq, H, hd = 4, lc.n_q_heads, lc.n_kv_heads, lc.head_dim
    width = -(-600 // P)
    perm = rng.permutation(N * width).reshape(N, width).tolist()
    kv, ref, lay = gpu_pages(lc, N * width, P, perm, 0x7F), P8.Pages(N * width, P, H, hd), handle(lc)
    length, live = [0] * N, {}
    for s, n_new in enumerate(steps):
        T = sum(n_new)
        x = rng.standard_normal((T, Hq + 2 * H, hd)) * np.exp(2.0 * rng.standard_normal((T, 1, 1))) * 4.0 ** (s % 3)
        x[rng.random(x.shape) < 0.01] = 0.0
        qkv = torch.tensor(x).to(tdtype(lc)).reshape(T, -1).to(DEV)
        slot = []
        for i, n in enumerate(n_new):
            for p in range(length[i], length[i] + n):
                slot.append(perm[i][p // P] * P + p % P)
                live[perm[i][p // P]] = p % P + 1
            length[i] += n
        rot = torch.zeros((T, hd // 2, 2), device=DEV)
        rot[..., 0] = 1.0
        q = torch.full((T, Hq * hd), float("nan"), dtype=tdtype(lc), device=DEV)
        lay.compact_rope_paged_write(qkv, kv, torch.tensor(slot, device=DEV), rot, q)
        y = f64(qkv).reshape(T, Hq + 2 * H, hd)
        ref.write(slot, y[:, Hq:Hq + H], y[:, Hq + H:])
        compare_pages(kv, ref, live)
        assert torch.equal(q, qkv[:, :Hq * hd])
    # rows behind the live ones are the earlier tenant's
    for page, n in live.items():
        assert (kv.k[page, :, n:] == 0x7F).all() and (kv.v[page, :, :, n:] == 0x7F).all()


@pytest.mark.parametrize("lc", [layer(2, 1, 64), layer(3, 3, 128), layer(2, 1, 64, "fp32")], ids=lambda c: "%d_%d_%s" % (c.n_kv_heads, c.head_dim, c.dtype))
@pytest.mark.parametrize("P", [16, 128])
@pytest.mark.parametrize("N,prompt", [(150, 0), (700, 300), (1000, 8000)])
def test_single_rows_among_others(lc, P, N, prompt):
    """A batch of mostly one row per request, at every place of a page, behind rows that are smaller, alike and larger (so that
    scales grow or stay), some rows not finite, segments of a few rows and a prompt among them."""
    if N > 700 and lc.head_dim == 128:
        pytest.skip("the same paths as with 700 requests; slow on the host")
    rng = np.random.default_rng(N + P)
    Hq, H, hd, dt = lc.n_q_heads, lc.n_kv_heads, lc.head_dim, tdtype(lc)
    before = rng.integers(0, P, N)
    n_new = rng.choice([0, 1, 1, 1, 1, 1, 1, 2, 3, 5], N)
    before[N // 2], n_new[N // 2] = 0, prompt
    start = np.concatenate([[0], np.cumsum((before + n_new + P - 1) // P)])      # request i has pages start[i] ..
    kv, ref, lay = gpu_pages(lc, int(start[-1]), P, [[0]], 0x7F), P8.Pages(int(start[-1]), P, H, hd), handle(lc)
    live = {}
    for lo, n in ((np.zeros_like(before), before), (before, n_new)):
        T = int(n.sum())
        x = rng.standard_normal((T, Hq + 2 * H, hd)) * np.exp(1.5 * rng.standard_normal((T, 1, 1)))
        if lo is before:
            x[rng.random(T) < 0.1, Hq + H - 1, 5] = np.inf
            x[rng.random(T) < 0.1, Hq + 2 * H - 1, 60] = np.nan
        slot, at = np.full(T, -1), 0
        for i in range(N):
            rows = np.arange(lo[i], lo[i] + n[i])
            slot[at:at + n[i]] = start[i] * P + rows
            at += n[i]
            live.update({int(start[i] + r // P): int(r % P) + 1 for r in rows})
        qkv = torch.tensor(x).to(dt).reshape(T, -1).to(DEV)
        rot = torch.zeros((T, hd // 2, 2), device=DEV)
        rot[..., 0] = 1.0
        q = torch.empty((T, Hq * hd), dtype=dt, device=DEV)
        lay.compact_rope_paged_write(qkv, kv, torch.tensor(slot, device=DEV), rot, q)
        y = f64(qkv).reshape(T, Hq + 2 * H, hd)
        with np.errstate(invalid="ignore"):
            k = P8.rope(y[:, Hq:Hq + H], f64(rot))     # (an infinity times a sine of 0 breaks its partner too)
        ref.write(slot.tolist(), k, y[:, Hq + H:])
        assert torch.equal(q, qkv[:, :Hq * hd])
    compare_pages(kv, ref, live)
    for page, n in live.items():
        assert (kv.k[page, :, n:] == 0x7F).all() and (kv.v[page, :, :, n:] == 0x7F).all()


@pytest.mark.parametrize("lc", WRITE_LAYERS, ids=lambda c: "%d_%d_%d_%s" % (c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype))
def test_rotated_rows(lc):
    """q and K rotated at large positions: q to one rounding, a K code to half a step of its value."""
    rng = np.random.default_rng(3)
    T, P, Hq, H, hd = 77, 32, lc.n_q_heads, lc.n_kv_heads, lc.head_dim
    pos = np.arange(T) + 100000
    ang = pos[:, None] * lc.rope_theta ** (-np.arange(hd // 2) / (hd // 2))
    rot = torch.tensor(np.stack([np.cos(ang), np.sin(ang)], -1)).float().to(DEV)
    qkv = torch.tensor(rng.standard_normal((T, (Hq + 2 * H) * hd))).to(tdtype(lc)).to(DEV)
    kv = gpu_pages(lc, 3, P, [[2, 0, 1]], 0)
    slot = [[2, 0, 1][r // P] * P + r % P for r in range(T)]
    q = torch.empty((T, Hq * hd), dtype=tdtype(lc), device=DEV)
    handle(lc).compact_rope_paged_write(qkv, kv, torch.tensor(slot, device=DEV), rot, q)
    want = P8.rope(f64(qkv).reshape(T, Hq + 2 * H, hd)[:, :Hq + H], f64(rot))
    size = P8.rope(np.abs(f64(qkv).reshape(T, Hq + 2 * H, hd)[:, :Hq + H]), np.abs(f64(rot)) * np.array([1.0, 1.0]))
    size = np.maximum(size, np.abs(want)) + np.abs(f64(qkv).reshape(T, Hq + 2 * H, hd)[:, :Hq + H])
    half = 2.0 ** -8 if lc.dtype == "bf16" else 2.0 ** -24
    fp32 = 2.0 ** -22 * (np.abs(size) + np.roll(np.abs(size), hd // 2, -1))     # products and sum of a rotation in fp32
    assert (np.abs(f64(q).reshape(T, Hq, hd) - want[:, :Hq]) <= half * np.abs(want[:, :Hq]) * 1.001 + fp32[:, :Hq]).all()
    got_k, got_v = kv.rows(0, T)
    byte = kv.k_scale.cpu().numpy().astype(np.float64)
    step = np.array([2.0 ** (byte[[2, 0, 1][r // P]] - 127 - 10) for r in range(T)])[:, :, None]     # half the smallest code
    assert (np.abs(f64(got_k) - want[:, Hq:]) <= np.maximum(2.0 ** -4 * np.abs(want[:, Hq:]), step) * 1.001 + fp32[:, Hq:]).all()


def test_rotation_has_the_bits_of_the_slab_path():
    lc = layer(8, 2, 128, theta=500000.0)
    lay, T, P = handle(lc), 300, 64
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((T, 12 * 128), generator=g).bfloat16().to(DEV)
    kv = B.PagedKV.allocate(lc, 1, 8, 8, P, DEV)
    st = B.PagedStep(lc, 1, T, DEV, n_pages=8, n_new=ints([T]))
    lay.compact_paged_plan(kv, st)
    q = torch.empty((T, 8 * 128), dtype=torch.bfloat16, device=DEV)
    lay.compact_rope_paged_write(qkv, kv, st.slot, st.rot, q)
    slab, other = B.KVCache(lc, [T], DEV, torch.bfloat16), qkv.clone()
    lay.compact_rope_kvwrite([0, T], other, slab)
    assert torch.equal(q, other[:, :8 * 128])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 40])
def test_extreme_and_broken_values(dtype, T):
    """Zeros, the smallest and the largest values, infinities and NaN: scales from the finite values alone, a broken row's K
    is NaN in its head, what is broken of V is 0, and rows without a slot leave no trace."""
    lc = layer(2, 2, 64, dtype)
    big = float(torch.finfo(tdtype(lc)).max)
    P, N = 16, 8
    kv, ref, lay = gpu_pages(lc, 64, P, [[i] for i in range(64)], 0x55), P8.Pages(64, P, 2, 64), handle(lc)
    rng = np.random.default_rng(5)
    x = rng.standard_normal((T * N, 6, 64))
    kinds = [lambda y: y * 0.0, lambda y: y * 1e-38, lambda y: np.sign(y) * big, lambda y: y * 1e30]
    for r in range(T * N):
        x[r] = kinds[r % 4](x[r])
    x = f64(torch.tensor(x).to(tdtype(lc)))
    x[0, 2, 3], x[1, 4, 5], x[2, 3, 60], x[min(9, T * N - 1), 5, 0] = np.inf, -np.inf, np.nan, np.nan
    slot = [-1 if r % 7 == 6 else (r // P) * P + r % P for r in range(T * N)] if T > 1 else [r * P for r in range(N)]
    if T == 1:
        slot[5] = 64 * P          # past the last page: nowhere
    qkv = torch.tensor(x).to(tdtype(lc)).reshape(T * N, -1).to(DEV)
    rot = torch.zeros((T * N, 32, 2), device=DEV)
    rot[..., 0] = 1.0
    q = torch.empty((T * N, 128), dtype=tdtype(lc), device=DEV)
    # rows -1 cut pages into pieces: written piece by piece, as consecutive slots ask for
    if T > 1:
        for a in range(0, T * N, 7):
            lay.compact_rope_paged_write(qkv[a:a + 7], kv, torch.tensor(slot[a:a + 7], device=DEV), rot[a:a + 7], q[a:a + 7])
            ref.write(slot[a:a + 7], x[a:a + 7, 2:4], x[a:a + 7, 4:6])
    else:
        lay.compact_rope_paged_write(qkv, kv, torch.tensor(slot, device=DEV), rot, q)
        ref.write([-1 if s >= 64 * P else s for s in slot], x[:, 2:4], x[:, 4:6])
    written = {}
    for s in slot:
        if 0 <= s < 64 * P:
            written.setdefault(s // P, []).append(s % P)
    for page, rows in written.items():
        k, v = kv.k[page].cpu().numpy()[:, rows], kv.v[page].cpu().numpy()[:, :, rows]
        assert np.array_equal(kv.k_scale[page].cpu().numpy(), ref.scale["k"][page]) and np.array_equal(kv.v_scale[page].cpu().numpy(), ref.scale["v"][page])
        # (the rotation by nothing may turn a zero's sign)
        assert np.array_equal(P8.VALUES[k], P8.VALUES[ref.codes["k"][page, rows].transpose(1, 0, 2)], equal_nan=True)
        assert np.array_equal(v, ref.codes["v"][page, rows].transpose(1, 2, 0))
    for page in set(range(64)) - set(written):
        assert (kv.k[page] == 0x55).all() and (kv.v[page] == 0x55).all() and (kv.k_scale[page] == 0x55).all()


# ---- attention -----------------------------------------------------------------------------------------------------------

def random_cache(lc, lens, P, seed, extra=3, fill=0x7F):
    """Pages of random codes and scales at random places; what no request owns is NaN, codes and scales."""
    rng = np.random.default_rng(seed)
    width = max(1, max(-(-n // P) for n in lens)) + 2
    used = sum(-(-n // P) for n in lens)
    n_pages = used + extra
    perm = rng.permutation(n_pages)
    table, at = np.full((len(lens), width), -1), 0
    ref = P8.Pages(n_pages, P, lc.n_kv_heads, lc.head_dim)
    for n in "kv":
        ref.codes[n][:] = 0x7F if fill else 0
        ref.scale[n][:] = 255 if fill else 1
    for i, n in enumerate(lens):
        c = -(-n // P)
        table[i, :c] = perm[at:at + c]
        at += c
        for j in range(c):
            rows, page = min(P, n - j * P), table[i, j]
            for name in "kv":
                x = rng.standard_normal((rows, lc.n_kv_heads, lc.head_dim)) * np.exp(0.7 * rng.standard_normal())
                x[..., 5::31] *= 3.0
                e = rng.integers(-1, 2, lc.n_kv_heads)
                # codes of another scale than the least one: any scale may stand there
                byte = np.array([P8.scale_byte(np.abs(x[:, h]).max()) for h in range(lc.n_kv_heads)]) + np.maximum(e, 0)
                ref.scale[name][page] = byte
                ref.codes[name][page, :rows] = P8.to_e4m3(x / 2.0 ** (byte[None, :, None] - 127.0))
    kv = B.PagedKV.allocate(lc, len(lens), width, n_pages, P, DEV)
    kv.k.copy_(torch.from_numpy(ref.codes["k"].transpose(0, 2, 1, 3).copy()))
    kv.v.copy_(torch.from_numpy(ref.codes["v"].transpose(0, 2, 3, 1).copy()))
    kv.k_scale.copy_(torch.from_numpy(ref.scale["k"].astype(np.uint8)))
    kv.v_scale.copy_(torch.from_numpy(ref.scale["v"].astype(np.uint8)))
    kv.table.copy_(torch.from_numpy(table.astype(np.int32)))
    return kv, ref, table


def queries(lc, n, seed, stride=None):
    g = torch.Generator().manual_seed(seed)
    Dq = lc.n_q_heads * lc.head_dim
    q = torch.full((n, stride or Dq), float("nan"))
    q[:, :Dq] = torch.randn((n, Dq), generator=g)
    return q.to(tdtype(lc)).to(DEV)[:, :Dq]


def run_attn(lay, kv, q, n_new, kv_len, max_new=None, max_kv=None):
    cu = np.concatenate([[0], np.cumsum(n_new)]).tolist()
    o = torch.full((q.shape[0], lay.layer.n_q_heads * lay.layer.head_dim), 77.0, dtype=q.dtype, device=DEV)
    bounds = (max_new or max(max(n_new), 1), max_kv or max(max(kv_len), 1))
    lay.ensure_paged_workspace(len(n_new), q.shape[0], *bounds, DEV)
    lay.compact_attn_paged(q, kv, ints(cu), ints(kv_len), *bounds, o)
    return o


def check_attn(lc, q, o, n_new, kv_len, ref, table):
    """Each element within the roundings there are (bf16 has 8 significant bits: half a step is 2^-8).  With A = sum p |v|: a probability rounded to bf16 (fp32 storage: none),
    the output rounded once, and 2^-13 A (fp32 storage 2^-15 A) for the scores and sums in fp32."""
    Hq, hd, row = lc.n_q_heads, lc.head_dim, 0
    half, rest = (2.0 ** -8, 2.0 ** -13) if lc.dtype == "bf16" else (0.0, 2.0 ** -15)
    out = 2.0 ** -8 if lc.dtype == "bf16" else 2.0 ** -24
    for i, (n, L) in enumerate(zip(n_new, kv_len)):
        if n:
            k, v = ref.rows("k", table[i], L), ref.rows("v", table[i], L)
            x = f64(q[row:row + n]).reshape(n, Hq, hd)
            want, size = P8.attend(x, k, v), P8.attend(x, k, np.abs(v))
            got = f64(o[row:row + n]).reshape(n, Hq, hd)
            assert np.array_equal(np.isnan(got), np.isnan(want)), i
            off = np.abs(got - want) - (half * size + out * np.abs(want) * 1.01 + rest * size)
            assert np.nanmax(off, initial=-1.0) <= 0, (i, n, L, np.nanmax(np.abs(got - want)), np.unravel_index(np.nanargmax(off), off.shape))
        row += n


ATTN_LAYERS = [layer(32, 8, 128), layer(16, 2, 64), layer(5, 5, 128), layer(16, 1, 64), layer(10, 2, 128), layer(9, 3, 64),
               layer(4, 2, 64, "fp32"), layer(6, 1, 128, "fp32")]
IDS = lambda c: "%d_%d_%d_%s" % (c.n_q_heads, c.n_kv_heads, c.head_dim, c.dtype)   # noqa: E731


@pytest.mark.parametrize("lc", ATTN_LAYERS, ids=IDS)
@pytest.mark.parametrize("P", [16, 64, 128])
def test_single_tokens(lc, P):
    """Lengths around pages, granules and pieces, a request that rests (length 0: zeros) and one with a row of its own only."""
    lens = [1, 2, 15, 16, 17, 0, 63, 64, 65, 129, 255, 256, 257, 511, 513, 1100]
    kv, ref, table = random_cache(lc, lens, P, P)
    q, lay = queries(lc, len(lens), P), handle(lc)
    o = run_attn(lay, kv, q, [1] * len(lens), lens)
    assert (o[5] == 0).all()
    check_attn(lc, q, o, [1] * len(lens), lens, ref, table)


@pytest.mark.parametrize("lc", ATTN_LAYERS, ids=IDS)
@pytest.mark.parametrize("P", [16, 32, 128])
def test_prompts_and_chunks(lc, P):
    """Whole prompts, chunks behind cached rows, a few rows to verify, single tokens and no rows at all in one call."""
    n_new = [1, 2, 3, 0, 5, 17, 33, 64, 65, 130, 1, 200]
    lens = [300, 2, 40, 77, 600, 17, 1500, 64, 70, 1030, 0, 333]
    kv, ref, table = random_cache(lc, lens, P, P + 1)
    q, lay = queries(lc, sum(n_new), P + 1), handle(lc)
    check_attn(lc, q, run_attn(lay, kv, q, n_new, lens), n_new, lens, ref, table)


@pytest.mark.parametrize("lc", [layer(8, 2, 128), layer(8, 1, 64), layer(4, 2, 64, "fp32")], ids=IDS)
def test_rows_that_see_nothing(lc):
    """More query rows than cached ones: the first rows see nothing and are zeros; kv_len 0: all of them."""
    n_new, lens = [3, 40, 200, 4], [1, 30, 0, 4]
    kv, ref, table = random_cache(lc, lens, 32, 4)
    q, lay = queries(lc, sum(n_new), 4), handle(lc)
    o = run_attn(lay, kv, q, n_new, lens)
    check_attn(lc, q, o, n_new, lens, ref, table)
    assert (o[0:2] == 0).all() and (o[3:13] == 0).all() and (o[43:243] == 0).all()


@pytest.mark.parametrize("lc", [layer(32, 8, 128), layer(64, 8, 64), layer(4, 2, 64, "fp32")], ids=IDS)
def test_long_caches(lc):
    """Keys split among many pieces, for single tokens and for tiles of rows."""
    n_new, lens = [1, 7, 40], [9000, 5001, 7777]
    kv, ref, table = random_cache(lc, lens, 64, 6)
    q, lay = queries(lc, sum(n_new), 6), handle(lc)
    check_attn(lc, q, run_attn(lay, kv, q, n_new, lens), n_new, lens, ref, table)


@pytest.mark.parametrize("lc", [layer(2, 2, 64), layer(2, 2, 128), layer(2, 2, 64, "fp32"), layer(8, 1, 64)], ids=IDS)
def test_long_chunks_in_pieces(lc):
    """Chunks of many rows whose keys are cut: rows that see nothing of a later piece, lengths around the cut, beside one that is not cut."""
    if lc.n_kv_heads == 2:
        n_new, lens = [2000, 4090, 300, 300, 1, 60], [4100, 4096, 4095, 4096, 4200, 1000]
    else:
        n_new, lens = [300, 40, 3], [6500, 4500, 4097]
    kv, ref, table = random_cache(lc, lens, 64, 16)
    q, lay = queries(lc, sum(n_new), 16), handle(lc)
    o = run_attn(lay, kv, q, n_new, lens)
    check_attn(lc, q, o, n_new, lens, ref, table)
    one = B.PagedKV(lc, kv.k, kv.v, kv.k_scale, kv.v_scale, kv.table[:1].contiguous())
    assert torch.equal(run_attn(lay, one, q[:n_new[0]], n_new[:1], lens[:1]), o[:n_new[0]])


@pytest.mark.parametrize("lc", [layer(8, 2, 128), layer(8, 2, 64), layer(4, 2, 64, "fp32")], ids=IDS)
def test_large_scores_and_growing_maxima(lc):
    """Scores in the hundreds that grow along the keys: the running maximum moves at nearly every step."""
    n_new, lens = [1, 50], [900, 800]
    kv, ref, table = random_cache(lc, lens, 64, 8)
    for i, n in enumerate(lens):
        for j in range(-(-n // 64)):
            ref.scale["k"][table[i][j]] += min(j, 8) // 2
    kv.k_scale.copy_(torch.from_numpy(ref.scale["k"].astype(np.uint8)))
    q, lay = queries(lc, sum(n_new), 8) * 4, handle(lc)
    o = run_attn(lay, kv, q, n_new, lens)
    # a score of size S carries 2^-22 S from its sum in fp32, so a probability as much of itself
    Hq, hd, row = lc.n_q_heads, lc.head_dim, 0
    for i, (n, L) in enumerate(zip(n_new, lens)):
        k, v = ref.rows("k", table[i], L), ref.rows("v", table[i], L)
        x = f64(q[row:row + n]).reshape(n, Hq, hd)
        want, size = P8.attend(x, k, v), P8.attend(x, k, np.abs(v))
        S = np.einsum("nhd,lhd->nhl", np.abs(x), np.abs(np.repeat(k, Hq // lc.n_kv_heads, 1))).max(-1, keepdims=True) / hd ** 0.5
        tol = (2.0 ** -8 if lc.dtype == "bf16" else 0) * (size + np.abs(want) * 1.01) + (2.0 ** -13 if lc.dtype == "bf16" else 2.0 ** -15) * size + 2.0 ** -21 * S * size
        # (a probability below 2^-126 is none in fp32)
        assert (np.abs(f64(o[row:row + n]).reshape(n, Hq, hd) - want) <= tol + 2.0 ** -126 * L * np.abs(v).max()).all()
        row += n


def test_a_broken_row_reaches_only_those_that_see_it():
    lc = layer(8, 2, 128)
    lay, P = handle(lc), 32
    for n_new, lens, broken in (([40], [40], 20), ([3], [300], 298), ([1], [300], 299), ([200], [600], 500)):
        T = lens[0]
        kv = B.PagedKV.allocate(lc, 1, 20, 20, P, DEV)
        for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
            t.fill_(0x7F)
        st = B.PagedStep(lc, 1, T, DEV, n_pages=20, n_new=ints([T]))
        lay.compact_paged_plan(kv, st)
        g = torch.Generator().manual_seed(2)
        qkv = torch.randn((T, 12 * 128), generator=g).bfloat16()
        qkv[broken, 11 * 128 + 7] = float("inf")           # V of KV head 1
        q = torch.empty((T, 8 * 128), dtype=torch.bfloat16, device=DEV)
        lay.compact_rope_paged_write(qkv.to(DEV), kv, st.slot, st.rot, q)
        n = n_new[0]
        o = run_attn(lay, kv, q[T - n:], n_new, lens).view(n, 8, 128)
        bad = torch.isnan(o)
        first = max(0, broken - (T - n))
        assert bad[first:, 4:].all() and not bad[:first].any() and not bad[:, :4].any()


@pytest.mark.parametrize("lc", [layer(32, 8, 128), layer(16, 2, 64), layer(4, 2, 64, "fp32")], ids=IDS)
def test_a_request_does_not_depend_on_the_others(lc):
    """The bits of a request alone, in a batch, at another place in it, and again."""
    n_new, lens = [1, 60, 3, 1, 130, 1], [2000, 2600, 700, 256, 130, 1]
    kv, ref, table = random_cache(lc, lens, 16, 9)
    q, lay = queries(lc, sum(n_new), 9), handle(lc)
    both = run_attn(lay, kv, q, n_new, lens)
    assert torch.equal(both, run_attn(lay, kv, q, n_new, lens, max_new=500, max_kv=30000))
    row = 0
    for i, (n, L) in enumerate(zip(n_new, lens)):
        one = B.PagedKV(lc, kv.k, kv.v, kv.k_scale, kv.v_scale, kv.table[i:i + 1].contiguous())
        assert torch.equal(run_attn(lay, one, q[row:row + n], [n], [L]), both[row:row + n]), i
        row += n
    back = B.PagedKV(lc, kv.k, kv.v, kv.k_scale, kv.v_scale, kv.table.flip(0).contiguous())
    rows = torch.split(q, n_new)
    got = run_attn(lay, back, torch.cat(rows[::-1]), n_new[::-1], lens[::-1])
    assert torch.equal(torch.cat(torch.split(got, n_new[::-1])[::-1]), both)


@pytest.mark.parametrize("lc", [layer(32, 8, 128), layer(16, 1, 128), layer(64, 8, 64), layer(9, 3, 64), layer(4, 2, 64, "fp32"), layer(6, 1, 128, "fp32")], ids=IDS)
@pytest.mark.parametrize("P", [16, 64])
def test_a_few_rows_behind_a_cache(lc, P):
    """Requests of one column to a few more than 32, by themselves (no prompt in the call: other kernels) and beside a prompt
    whose keys are split too; a call with none but few rows, and one with single rows among them."""
    G = lc.n_q_heads // lc.n_kv_heads
    n_new = sorted({1, 2, 15 // G + 1, 16 // G, 16 // G + 1, 31 // G + 1, 32 // G, 32 // G + 1} - {0}) + [40, 1]
    lens = [[3, 300, 513, 1500, 256, 257, 17, 700, 40, 2100][i % 10] for i in range(len(n_new))]
    lens[-2], lens[-1] = 2100, 900
    lens = [max(n, L) for n, L in zip(n_new, lens)]
    kv, ref, table = random_cache(lc, lens, P, P + G)
    q, lay = queries(lc, sum(n_new), P), handle(lc)
    both = run_attn(lay, kv, q, n_new, lens)
    check_attn(lc, q, both, n_new, lens, ref, table)
    rows, want = torch.split(q, n_new), torch.split(both, n_new)
    for least, most in ((1, 16 // G), (1, 32 // G), (2, 32 // G)):
        some = [i for i, n in enumerate(n_new) if least <= n <= most]
        if not some:
            continue
        sub = B.PagedKV(lc, kv.k, kv.v, kv.k_scale, kv.v_scale, kv.table[some].contiguous())
        got = run_attn(lay, sub, torch.cat([rows[i] for i in some]), [n_new[i] for i in some], [lens[i] for i in some])
        assert torch.equal(got, torch.cat([want[i] for i in some])), (least, most)


@pytest.mark.parametrize("N", [65, 300])
def test_many_requests_beside_a_prompt(N):
    """More requests than a wavefront looks at side by side, most of them single rows of split caches, some resting."""
    lc = layer(4, 2, 64)
    rng = np.random.default_rng(N)
    n_new = rng.choice([0, 1, 1, 1, 2, 20], N).tolist()
    lens = [max(n, int(L)) for n, L in zip(n_new, rng.integers(1, 700, N))]
    n_new[N // 2], lens[N // 2] = 90, 1100
    kv, ref, table = random_cache(lc, lens, 32, N)
    q, lay = queries(lc, sum(n_new), N), handle(lc)
    o = run_attn(lay, kv, q, n_new, [L if n else 0 for n, L in zip(n_new, lens)])
    check_attn(lc, q, o, n_new, lens, ref, table)


def test_strided_queries_and_rows_of_nobody():
    lc = layer(8, 2, 64)
    n_new, lens = [2, 30], [50, 400]
    kv, ref, table = random_cache(lc, lens, 16, 11)
    lay = handle(lc)
    q = queries(lc, 40, 11, stride=12 * 64 + 8)
    o = run_attn(lay, kv, q, n_new, lens)
    check_attn(lc, q, o, n_new, lens, ref, table)
    assert (o[32:] == 77.0).all()


def test_table_entries_and_lengths_out_of_range_stay_inside_the_buffers():
    """Nothing is promised for such a request's rows, but the others' are right and nothing is read outside the pages (their
    numbers are brought into range by the kernels)."""
    lc = layer(8, 2, 128)
    n_new, lens = [1, 40, 1, 40], [300, 300, 300, 300]
    kv, ref, table = random_cache(lc, lens, 64, 12)
    kv.table[0, 1], kv.table[1, 2] = 1 << 30, -5
    q, lay = queries(lc, sum(n_new), 12), handle(lc)
    cu, said = ints([0, 1, 41, 42, 82]), ints([300, 300, 300, 300])
    o = torch.zeros_like(q)
    lay.ensure_paged_workspace(4, 82, 40, 300, DEV)
    lay.compact_attn_paged(q, kv, cu, said, 40, 300, o)
    for i, r in ((2, slice(41, 42)), (3, slice(42, 82))):
        check_attn(lc, q[r], o[r], [n_new[i]], [300], ref, table[i:i + 1])
    said[0], cu[1:] = 1 << 30, ints([1, 41, 42, 1 << 30])      # clamped to max_kv_len and to the rows there are
    lay.compact_attn_paged(q, kv, cu, said, 40, 300, o)
    check_attn(lc, q[41:42], o[41:42], [1], [300], ref, table[2:3])


def test_pages_beyond_4_gib():
    """Offsets that pass 32 bits, into the codes and into a pool of more than 2^31 rows' elements."""
    lc = layer(8, 8, 128)
    P, n_pages = 128, 36000                              # 128 KiB a page: 4.7 GB of K codes
    lay = handle(lc)
    kv = B.PagedKV.allocate(lc, 2, 4, n_pages, P, DEV)
    st = B.PagedStep(lc, 2, 300, DEV, n_new=ints([260, 40]), free=torch.arange(n_pages, dtype=torch.int32, device=DEV))   # the last pages first
    lay.compact_paged_plan(kv, st)
    assert kv.table[0, 0].item() == n_pages - 1
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((300, 24 * 128), generator=g).bfloat16().to(DEV)
    q = torch.empty((300, 8 * 128), dtype=torch.bfloat16, device=DEV)
    lay.compact_rope_paged_write(qkv, kv, st.slot, st.rot, q)
    small = B.PagedKV.allocate(lc, 2, 4, 6, P, DEV)
    st2 = B.PagedStep(lc, 2, 300, DEV, n_pages=6, n_new=ints([260, 40]))
    lay.compact_paged_plan(small, st2)
    lay.compact_rope_paged_write(qkv, small, st2.slot, st2.rot, torch.empty_like(q))
    for n_new, rows in (([260, 40], q), ([1, 1], q[[259, 299]].contiguous())):
        assert torch.equal(run_attn(lay, kv, rows, n_new, [260, 40]), run_attn(lay, small, rows, n_new, [260, 40]))


# ---- together ------------------------------------------------------------------------------------------------------------

def test_decode_steps_from_a_graph():
    """Plan, write and attention of a step captured once and replayed: every step as it comes out of eager calls, with other
    work between the replays.  Lengths and stacks swap places, so two steps are one graph."""
    lc = layer(8, 2, 64)
    lay, N, P = handle(lc), 6, 16
    g = torch.Generator().manual_seed(4)
    x = torch.randn((40, N, 12 * 64), generator=g).bfloat16().to(DEV)

    def fresh():
        kv = B.PagedKV.allocate(lc, N, 8, 40, P, DEV)
        for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
            t.zero_()
        return kv, B.PagedStep(lc, N, N, DEV, n_pages=40, n_new=ints([1, 1, 0, 1, 1, 1]))

    def step(kv, st, qkv, q, o):
        lay.compact_paged_plan(kv, st)
        lay.compact_rope_paged_write(qkv, kv, st.slot, st.rot, q)
        lay.compact_attn_paged(q, kv, st.cu, st.kv_len, 1, 128, o)
        st.advance()

    lay.ensure_paged_workspace(N, N, 1, 128, DEV)
    bufs = [[torch.zeros((N, 12 * 64), dtype=torch.bfloat16, device=DEV)] + [torch.zeros((N, 8 * 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            for _ in range(2)]
    kv, st = fresh()
    eager = []
    for s in range(40):
        bufs[0][0].copy_(x[s])
        step(kv, st, *bufs[0])
        eager.append(bufs[0][2].clone())
    kv, st = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for b in bufs:
            step(kv, st, *b)
    for s in range(0, 40, 2):
        bufs[0][0].copy_(x[s])
        bufs[1][0].copy_(x[s + 1])
        graph.replay()
        assert torch.equal(bufs[0][2], eager[s]) and torch.equal(bufs[1][2], eager[s + 1]), s
        torch.randn(1000, device=DEV).sum().item()
    assert st.len.tolist() == [40, 40, 0, 40, 40, 40]


def test_on_another_stream():
    lc = layer(8, 2, 64)
    n_new, lens = [1, 30], [700, 1500]
    kv, ref, table = random_cache(lc, lens, 32, 13)
    q, lay = queries(lc, 31, 13), handle(lc)
    want = run_attn(lay, kv, q, n_new, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run_attn(lay, kv, q, n_new, lens)
    side.synchronize()
    assert torch.equal(got, want)
