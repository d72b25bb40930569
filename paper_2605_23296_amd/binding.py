"""ctypes binding over libcompact.so: argument marshalling only.

The functions keep the names of the C ABI (include/compact.h).  `Layer` is a
thin convenience holder that owns torch-allocated device buffers (KV slabs,
workspace) and passes their addresses down; every step of the computation
runs in the library's kernels.  There is no fallback: if the library has not
been built, `lib()` raises.
"""
import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcompact.so")

COMPACT_FP32, COMPACT_BF16 = 0, 1
K_NONE, K_GEMM, K_ATTN_PREFILL, K_ATTN_DECODE, K_GEMM_SKINNY = 0, 1, 2, 3, 4
ERR_NAMES = {0: "OK", 1: "EINVAL", 2: "ESHAPE", 3: "ECAPACITY", 4: "EWORKSPACE", 5: "EUNSUPPORTED", 6: "EHIP"}

EXPORTS = [
    "compact_create", "compact_destroy", "compact_last_error", "compact_workspace_bytes",
    "compact_prefill", "compact_decode_step", "compact_layer_forward",
    "compact_profile_select", "compact_profile_read",
    "compact_rmsnorm", "compact_rope_kvwrite", "compact_gemm", "compact_attn_prefill",
    "compact_attn_decode", "compact_attn_decode_noalloc", "compact_moe_route", "compact_moe_ffn",
    "compact_prefix_workspace_bytes", "compact_prefix_decode_step", "compact_attn_decode_prefix",
    "compact_stack_workspace_bytes", "compact_stack_forward", "compact_prefill_extend", "compact_mxfp4_dequant",
    "compact_mixed_workspace_bytes", "compact_mixed_forward",
    "compact_prefix_stack_workspace_bytes", "compact_prefix_stack_forward",
    "compact_paged_plan", "compact_rope_paged_write", "compact_paged_workspace_bytes", "compact_attn_paged",
    "compact_quant_i8", "compact_gemm_i8_workspace_bytes", "compact_gemm_i8", "compact_block_norm", "compact_route",
    "compact_moe_ffn_i8_workspace_bytes", "compact_moe_ffn_i8",
]


class LayerCfg(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("ffn_dim", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("dtype", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("g_attn", "w_qkv", "w_o", "g_ffn", "w_gate_up", "w_down",
                                          "w_router", "w_exp_gate_up", "w_exp_down",
                                          "w_exp_gate_up_q", "w_exp_gate_up_s", "w_exp_down_q", "w_exp_down_s")]


class KV(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("h_slab_offset", C.POINTER(C.c_int64)), ("h_capacity", C.POINTER(C.c_int32)),
                ("h_len", C.POINTER(C.c_int32)), ("h_pos_offset", C.POINTER(C.c_int32))]


class RouteOut(C.Structure):
    _fields_ = [("d_expert_idx", C.c_void_p), ("d_gate", C.c_void_p)]


class PagedKVStruct(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_k_scale", C.c_void_p), ("d_v_scale", C.c_void_p), ("d_table", C.c_void_p),
                ("n_pages", C.c_int32), ("page_rows", C.c_int32), ("max_pages", C.c_int32), ("n_requests", C.c_int32)]


class PagedStepStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_n_new", "d_len", "d_n_free", "d_free", "d_n_free_out", "d_n_refused", "d_len_out",
                                          "d_kv_len", "d_cu", "d_slot", "d_rot")] + [("max_rows", C.c_int32)]


MAX_INT = 0x7fffffff   # (a 32-bit argument takes a larger number modulo 2^32, without a word)


class RouteRuleStruct(C.Structure):
    _fields_ = [("score", C.c_int32), ("n_groups", C.c_int32), ("topk_groups", C.c_int32), ("group_top", C.c_int32), ("renorm", C.c_int32),
                ("factor", C.c_float)]


class ExpertsI8Struct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_gate_up", "d_gate_up_scale", "d_down", "d_down_scale")]


class CompactError(RuntimeError):
    def __init__(self, code, detail):
        super().__init__("libcompact: %s (%d): %s" % (ERR_NAMES.get(code, "?"), code, detail))
        self.code = code
        self.detail = detail


_lib = None


def lib():
    """Loads libcompact.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libcompact.so is not built: run `python -m paper_2605_23296_amd.build` "
                           "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    P = C.POINTER
    L.compact_create.argtypes = [P(LayerCfg), P(vp)]
    L.compact_destroy.argtypes = [vp]
    L.compact_destroy.restype = None
    L.compact_last_error.argtypes = [vp]
    L.compact_last_error.restype = C.c_char_p
    L.compact_workspace_bytes.argtypes = [vp, i64, i32, i32, P(sz)]
    L.compact_prefill.argtypes = [vp, P(Weights), i32, P(i32), vp, P(KV), vp, P(RouteOut), vp, sz, vp]
    L.compact_decode_step.argtypes = [vp, P(Weights), i32, vp, P(KV), vp, P(RouteOut), vp, sz, vp]
    L.compact_prefill_extend.argtypes = [vp, P(Weights), i32, P(i32), vp, P(KV), vp, P(RouteOut), vp, sz, vp]
    L.compact_layer_forward.argtypes = [vp, P(Weights), i32, P(i32), vp, i32, vp, P(KV), vp, vp, vp, vp, sz, vp]
    L.compact_profile_select.argtypes = [vp, i32]
    L.compact_profile_read.argtypes = [vp, P(i64), P(C.c_double)]
    L.compact_rmsnorm.argtypes = [vp, vp, vp, vp, i64, vp]
    L.compact_rope_kvwrite.argtypes = [vp, i32, P(i32), vp, P(KV), vp]
    L.compact_gemm.argtypes = [vp, vp, vp, vp, vp, i64, i32, i32, i32, vp, sz, vp]
    L.compact_attn_prefill.argtypes = [vp, i32, P(i32), vp, P(KV), vp, vp]
    L.compact_attn_decode.argtypes = [vp, i32, vp, P(KV), vp, vp, sz, vp]
    L.compact_moe_route.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    L.compact_moe_ffn.argtypes = [vp, P(Weights), vp, vp, vp, vp, i64, vp, vp, sz, vp]
    L.compact_prefix_workspace_bytes.argtypes = [vp, i32, i32, i32, P(sz)]
    L.compact_prefix_decode_step.argtypes = [vp, P(Weights), i32, vp, P(KV), P(i32), P(KV), vp, P(RouteOut), vp, sz, vp]
    L.compact_attn_decode_prefix.argtypes = [vp, i32, vp, P(KV), P(i32), P(KV), vp, vp, sz, vp]
    L.compact_mixed_workspace_bytes.argtypes = [vp, i32, i32, i32, P(sz)]
    L.compact_mixed_forward.argtypes = [vp, P(Weights), i32, P(i32), vp, i32, vp, P(KV), i32, vp, vp, vp, sz, vp]
    L.compact_prefix_stack_workspace_bytes.argtypes = [vp, i64, i32, i32, P(sz)]
    L.compact_prefix_stack_forward.argtypes = [vp, i32, P(Weights), i32, P(i32), i64, vp, i32, vp, P(KV), P(KV), vp, vp, sz, vp]
    L.compact_mxfp4_dequant.argtypes = [vp, vp, vp, i64, i32, vp, vp]
    L.compact_stack_workspace_bytes.argtypes = [vp, i64, i32, i32, P(sz)]
    L.compact_stack_forward.argtypes = [vp, i32, P(Weights), i32, P(i32), vp, i32, vp, P(KV), vp, vp, vp, sz, vp]
    L.compact_paged_plan.argtypes = [vp, P(PagedKVStruct), P(PagedStepStruct), vp]
    L.compact_rope_paged_write.argtypes = [vp, i32, vp, P(PagedKVStruct), vp, vp, vp, vp]
    L.compact_paged_workspace_bytes.argtypes = [vp, i32, i32, i32, i32, P(sz)]
    L.compact_attn_paged.argtypes = [vp, P(PagedKVStruct), i32, vp, vp, i32, i32, vp, i64, vp, vp, sz, vp]
    L.compact_quant_i8.argtypes = [vp, vp, i64, i64, i32, vp, vp, vp]
    L.compact_gemm_i8_workspace_bytes.argtypes = [vp, i64, i32, i32, i32, P(sz)]
    L.compact_gemm_i8.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, vp, sz, vp]
    L.compact_block_norm.argtypes = [vp, vp, vp, vp, vp, i64, C.c_float, vp, vp, vp, vp, vp, i64, vp]
    L.compact_route.argtypes = [vp, P(RouteRuleStruct), vp, vp, vp, vp, i64, vp, vp, vp]
    L.compact_moe_ffn_i8_workspace_bytes.argtypes = [vp, i64, P(sz)]
    L.compact_moe_ffn_i8.argtypes = [vp, P(ExpertsI8Struct), vp, vp, vp, vp, vp, i64, vp, vp, sz, vp]
    for name in EXPORTS:
        fn = getattr(L, name)
        if name not in ("compact_destroy", "compact_last_error"):
            fn.restype = C.c_int
    _lib = L
    return L


def _ptr(t):
    if t is None:
        return None
    assert t.is_contiguous()
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _refuse(detail):
    raise CompactError(1, detail)


def _array(t, dtype, n, device, name):
    """Address of an array of at least n elements that a kernel on `device` may use as they lie there."""
    if t.dtype is not dtype or t.numel() < n or t.get_device() != device or not t.is_contiguous():
        _refuse("%s: %s %s on %s%s; contiguous %s, at least %d elements, on the current GPU needed"
                % (name, t.dtype, tuple(t.shape), t.device, "" if t.is_contiguous() else ", not contiguous", dtype, n))
    return t.data_ptr()


def _raw_stream(device):
    try:      # (0.1 us; the public way takes 2.7, half of a small call)
        return torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:
        return torch.cuda.current_stream(device).cuda_stream


def _i32arr(vals):
    return (C.c_int32 * len(vals))(*[int(v) for v in vals])


def make_cfg(layer):
    """layer: workloads.LayerConfig (or any object with the same fields)."""
    return LayerCfg(layer.d_model, layer.n_q_heads, layer.n_kv_heads, layer.head_dim, layer.ffn_dim,
                    layer.n_experts, layer.top_k, layer.rms_eps, layer.rope_theta,
                    COMPACT_BF16 if layer.dtype == "bf16" else COMPACT_FP32)


class KVCache:
    """Torch-allocated K/V slabs for N blocks plus the host arrays of compact_kv."""

    def __init__(self, layer, capacities, device, dtype, pos_offset=None):
        self.N = len(capacities)
        caps = [(int(c) + 7) // 8 * 8 for c in capacities]
        per_tok = layer.n_kv_heads * layer.head_dim
        offs, total = [], 0
        for c in caps:
            offs.append(total)
            total += c * per_tok
        self.k = torch.empty(max(total, 8), dtype=dtype, device=device)
        self.v = torch.empty(max(total, 8), dtype=dtype, device=device)
        self.h_slab_offset = (C.c_int64 * self.N)(*offs)
        self.h_capacity = _i32arr(caps)
        self.h_len = _i32arr([0] * self.N)
        self.h_pos_offset = None if pos_offset is None else _i32arr(pos_offset)
        self.layer = layer
        self.caps, self.offs = caps, offs
        self.c = KV(self.k.data_ptr(), self.v.data_ptr(), self.h_slab_offset, self.h_capacity, self.h_len,
                    self.h_pos_offset if self.h_pos_offset is not None else C.cast(None, C.POINTER(C.c_int32)))

    def lens(self):
        return [int(v) for v in self.h_len]

    def block_k(self, b):
        """K rows of block b as [len, Hkv, hd]."""
        L, Hkv, hd = self.h_len[b], self.layer.n_kv_heads, self.layer.head_dim
        slab = self.k[self.offs[b]:self.offs[b] + self.caps[b] * Hkv * hd].view(Hkv, self.caps[b], hd)
        return slab[:, :L, :].permute(1, 0, 2)

    def block_v(self, b):
        """V rows of block b as [len, Hkv, hd] (the slab stores them transposed)."""
        L, Hkv, hd = self.h_len[b], self.layer.n_kv_heads, self.layer.head_dim
        slab = self.v[self.offs[b]:self.offs[b] + self.caps[b] * Hkv * hd].view(Hkv, hd, self.caps[b])
        return slab[:, :, :L].permute(2, 0, 1)


class PagedKV:
    """Pages in 8 bits and their block table (compact_paged_kv): k uint8 [n_pages, Hkv, page_rows, hd], v uint8 [n_pages, Hkv,
    hd, page_rows], k_scale and v_scale uint8 [n_pages, Hkv], table int32 [n_requests, max_pages].  n_pages and page_rows
    are taken from k unless given (a plan needs the table alone).  The arrays may be replaced (a larger pool: k, v, both scales and
    n_pages); the next call uses the new ones."""

    def __init__(self, layer, k, v, k_scale, v_scale, table, n_pages=None, page_rows=None):
        self.layer, self.k, self.v, self.k_scale, self.v_scale, self.table = layer, k, v, k_scale, v_scale, table
        self.n_pages = k.shape[0] if n_pages is None else n_pages
        self.page_rows = k.shape[2] if page_rows is None else page_rows
        self.struct()

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_ref", None)   # (made again by the next call)

    def struct(self):
        """Reference to the compact_paged_kv of the arrays as they are."""
        if self._ref is None:
            layer, table, names = self.layer, self.table, ("k", "v", "k_scale", "v_scale")
            arrays = [getattr(self, name) for name in names]
            if self.k.numel():
                pages, rows = (self.n_pages, layer.n_kv_heads), (self.page_rows, layer.head_dim)
                for name, x, shape in zip(names, arrays, (pages + rows, pages + rows[::-1], pages, pages)):
                    if tuple(x.shape) != shape:
                        _refuse("pages: %s is %s, %s needed" % (name, tuple(x.shape), shape))
            device = table.get_device()
            for name, x in zip(names, arrays):
                _array(x, torch.uint8, 0, device, "pages: " + name)
            _array(table, torch.int32, 0, device, "block table")
            n_requests, max_pages = table.shape
            c = PagedKVStruct(*[x.data_ptr() for x in arrays], table.data_ptr(), self.n_pages, self.page_rows, max_pages, n_requests)
            for name, value in (("n_requests", n_requests), ("max_pages", max_pages), ("device", device),
                                ("heads", (layer.n_kv_heads, layer.head_dim)), ("c", c), ("_ref", C.byref(c))):
                object.__setattr__(self, name, value)
        return self._ref

    @classmethod
    def allocate(cls, layer, n_requests, max_pages, n_pages, page_rows, device):
        def pool(*shape):
            return torch.empty((n_pages, layer.n_kv_heads) + shape, dtype=torch.uint8, device=device)
        table = torch.full((n_requests, max_pages), -1, dtype=torch.int32, device=device)
        return cls(layer, pool(page_rows, layer.head_dim), pool(layer.head_dim, page_rows), pool(), pool(), table)

    def rows(self, request, length):
        """Cached rows of a request as fp32 [length, Hkv, hd] (K, V): the values that the codes stand for."""
        pages = self.table[request, :-(-length // self.page_rows)].long()

        def values(codes, scale):
            return codes[pages].view(torch.float8_e4m3fn).float() * scale[pages].view(torch.float8_e8m0fnu).float()[..., None, None]

        def flat(x):   # [pages, Hkv, page_rows, hd]
            return x.transpose(1, 2).reshape(-1, *x.shape[1:2], x.shape[3])[:length]
        return flat(values(self.k, self.k_scale)), flat(values(self.v, self.v_scale).transpose(2, 3))


class PagedStep:
    """Device arrays of a step's plan (compact_paged_step).  Arrays not given are allocated: all pages free, no rows cached."""

    def __init__(self, layer, n_requests, max_rows, device, n_pages=None, n_new=None, len=None, free=None, n_free=None):
        def ints(n, given=None):
            return torch.zeros(n, dtype=torch.int32, device=device) if given is None else given
        self.n_new, self.len = ints(n_requests, n_new), ints(n_requests, len)
        # the last entry of the stack is taken first: page 0
        self.free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device) if free is None else free
        self.n_free = ints(1, n_free) if n_free is not None else torch.tensor([self.free.numel()], dtype=torch.int32, device=device)
        self.n_free_out, self.n_refused = ints(1), ints(1)
        self.len_out, self.kv_len, self.cu = ints(n_requests), ints(n_requests), ints(n_requests + 1)
        self.slot = torch.empty(max_rows, dtype=torch.int64, device=device)
        self.rot = torch.empty((max_rows, layer.head_dim // 2, 2), dtype=torch.float32, device=device)
        self.n_requests, self.max_rows, self.head_dim = n_requests, max_rows, layer.head_dim

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_c", None)   # (made again by the next call)

    def struct(self):
        if self._c is None:
            N, i32, device = self.n_requests, torch.int32, self.n_new.get_device()
            if self.n_new.numel() != N or self.len.numel() != N:
                _refuse("step: %d requests, n_new of %d, len of %d" % (N, self.n_new.numel(), self.len.numel()))
            arrays = (("n_new", i32, N), ("len", i32, N), ("n_free", i32, 1), ("free", i32, 0), ("n_free_out", i32, 1), ("n_refused", i32, 1),
                      ("len_out", i32, N), ("kv_len", i32, N), ("cu", i32, N + 1), ("slot", torch.int64, self.max_rows),
                      ("rot", torch.float32, self.max_rows * self.head_dim))
            c = PagedStepStruct(*[_array(getattr(self, name), dtype, n, device, "step: " + name) for name, dtype, n in arrays], self.max_rows)
            for name, value in (("device", device), ("n_stack", self.free.numel()), ("_c", c)):
                object.__setattr__(self, name, value)
        return self._c

    def advance(self):
        """After a step: its lengths and its stack are the next one's."""
        c = self._c
        self.len, self.len_out = self.len_out, self.len
        self.n_free, self.n_free_out = self.n_free_out, self.n_free
        if c is not None:      # (the arrays are the same ones, and have been looked at)
            c.d_len, c.d_len_out, c.d_n_free, c.d_n_free_out = c.d_len_out, c.d_len, c.d_n_free_out, c.d_n_free
            object.__setattr__(self, "_c", c)


class RouteRule:
    """How compact_route chooses (compact_route_rule): score "softmax" or "sigmoid"; n_groups groups of experts of which topk_groups (None: all)
    are eligible, ranked by the sum of their group_top best; renorm divides the weights by their sum, factor multiplies them."""

    def __init__(self, score="softmax", n_groups=1, topk_groups=None, group_top=1, renorm=True, factor=1.0):
        if score not in ("softmax", "sigmoid"):
            _refuse("route: score %r; softmax or sigmoid needed" % (score,))
        if max(n_groups, topk_groups or 0, group_top) > MAX_INT or min(n_groups, topk_groups or 0, group_top) < 0:
            _refuse("route: %d groups, %s of them, %d experts of each; counts needed" % (n_groups, topk_groups, group_top))
        self.c = RouteRuleStruct(int(score == "sigmoid"), n_groups, n_groups if topk_groups is None else topk_groups, group_top, bool(renorm), factor)
        self.ref = C.byref(self.c)


class ExpertsI8:
    """Expert weights as codes (compact_experts_i8): gate_up int8 [E, 2F, d], gate_up_scale fp32 [E, 2F], down int8 [E, d, F], down_scale [E, d]."""

    def __init__(self, gate_up, gate_up_scale, down, down_scale):
        self.gate_up, self.gate_up_scale, self.down, self.down_scale = gate_up, gate_up_scale, down, down_scale


class Layer:
    """One layer context plus its weight pointers."""

    def __init__(self, layer, weights):
        self.L = lib()
        self.layer = layer
        self.cfg = make_cfg(layer)
        self.ctx = C.c_void_p()
        rc = self.L.compact_create(C.byref(self.cfg), C.byref(self.ctx))
        if rc != 0:
            raise CompactError(rc, self.L.compact_last_error(None).decode())
        self.weights = weights          # keeps the tensors alive
        self.w = Weights()
        for name, _ in Weights._fields_:
            t = weights.get(name) if weights is not None else None
            setattr(self.w, name, t.data_ptr() if t is not None else None)
        self.ws = None
        self.torch_dtype = torch.bfloat16 if layer.dtype == "bf16" else torch.float32
        self.kv_heads, self.d_model, self.experts = (layer.n_kv_heads, layer.head_dim), layer.d_model, (layer.n_experts, layer.top_k)
        self.q_cols, self.qkv_cols = layer.n_q_heads * layer.head_dim, (layer.n_q_heads + 2 * layer.n_kv_heads) * layer.head_dim

    def close(self):
        if self.ctx:
            self.L.compact_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def check(self, rc):
        if rc != 0:
            raise CompactError(rc, self.L.compact_last_error(self.ctx).decode())

    # -- workspace ------------------------------------------------------------
    def workspace_bytes(self, max_tokens, max_blocks, max_kv_len):
        n = C.c_size_t()
        self.check(self.L.compact_workspace_bytes(self.ctx, max_tokens, max_blocks, max_kv_len, C.byref(n)))
        return n.value

    def ensure_workspace(self, max_tokens, max_blocks, max_kv_len, device):
        need = self.workspace_bytes(max_tokens, max_blocks, max_kv_len)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        return self.ws

    def _ws(self):
        return (C.c_void_p(self.ws.data_ptr()), self.ws.numel()) if self.ws is not None else (None, 0)

    # -- layer calls ------------------------------------------------------------
    def compact_prefill(self, cu_seqlens, x, kv, y, route=None):
        wsp, wsn = self._ws()
        r = None if route is None else C.byref(RouteOut(route[0].data_ptr(), route[1].data_ptr()))
        self.check(self.L.compact_prefill(self.ctx, C.byref(self.w), len(cu_seqlens) - 1, _i32arr(cu_seqlens),
                                          _ptr(x), C.byref(kv.c), _ptr(y), r, wsp, wsn, _stream()))

    def compact_prefill_extend(self, cu_seqlens, x, kv, y, route=None):
        wsp, wsn = self._ws()
        r = None if route is None else C.byref(RouteOut(route[0].data_ptr(), route[1].data_ptr()))
        self.check(self.L.compact_prefill_extend(self.ctx, C.byref(self.w), len(cu_seqlens) - 1, _i32arr(cu_seqlens),
                                                 _ptr(x), C.byref(kv.c), _ptr(y), r, wsp, wsn, _stream()))

    def compact_decode_step(self, x, kv, y, route=None):
        wsp, wsn = self._ws()
        r = None if route is None else C.byref(RouteOut(route[0].data_ptr(), route[1].data_ptr()))
        self.check(self.L.compact_decode_step(self.ctx, C.byref(self.w), kv.N, _ptr(x), C.byref(kv.c), _ptr(y),
                                              r, wsp, wsn, _stream()))

    def compact_layer_forward(self, cu_seqlens, x_prefill, x_decode, kv, y_prefill, y_last, y_decode):
        wsp, wsn = self._ws()
        S = 0 if x_decode is None else x_decode.shape[0]
        self.check(self.L.compact_layer_forward(
            self.ctx, C.byref(self.w), len(cu_seqlens) - 1, _i32arr(cu_seqlens), _ptr(x_prefill), S,
            _ptr(x_decode), C.byref(kv.c), _ptr(y_prefill), _ptr(y_last), _ptr(y_decode), wsp, wsn, _stream()))

    # -- mixed batches (chunked prefill interleaved with decode) --------------------
    def mixed_workspace_bytes(self, max_batched_tokens, max_blocks, max_kv_len):
        n = C.c_size_t()
        self.check(self.L.compact_mixed_workspace_bytes(self.ctx, max_batched_tokens, max_blocks, max_kv_len, C.byref(n)))
        return n.value

    def compact_mixed_forward(self, cu_seqlens, x_prefill, x_decode, kv, max_batched_tokens, y_last, y_decode):
        wsp, wsn = self._ws()
        S = 0 if x_decode is None else x_decode.shape[0]
        self.check(self.L.compact_mixed_forward(
            self.ctx, C.byref(self.w), len(cu_seqlens) - 1, _i32arr(cu_seqlens), _ptr(x_prefill), S, _ptr(x_decode),
            C.byref(kv.c), max_batched_tokens, _ptr(y_last), _ptr(y_decode), wsp, wsn, _stream()))

    # -- a depth of layers --------------------------------------------------------
    def stack_workspace_bytes(self, max_tokens, max_blocks, max_kv_len):
        n = C.c_size_t()
        self.check(self.L.compact_stack_workspace_bytes(self.ctx, max_tokens, max_blocks, max_kv_len, C.byref(n)))
        return n.value

    def compact_stack_forward(self, layer_weights, cu_seqlens, x_prefill, x_decode, kvs, y_last, y_decode):
        """layer_weights: one dict of device tensors per layer; kvs: one KVCache per layer (same geometry)."""
        wsp, wsn = self._ws()
        nl = len(layer_weights)
        warr = (Weights * nl)()
        for l, wd in enumerate(layer_weights):
            for name, _ in Weights._fields_:
                t = wd.get(name)
                setattr(warr[l], name, t.data_ptr() if t is not None else None)
        karr = (KV * nl)()
        for l, kv in enumerate(kvs):
            for name, _ in KV._fields_:
                setattr(karr[l], name, getattr(kv.c, name))
        S = 0 if x_decode is None else x_decode.shape[0]
        self.check(self.L.compact_stack_forward(
            self.ctx, nl, warr, len(cu_seqlens) - 1, _i32arr(cu_seqlens), _ptr(x_prefill), S, _ptr(x_decode), karr,
            _ptr(y_last), _ptr(y_decode), wsp, wsn, _stream()))

    def prefix_stack_workspace_bytes(self, history_tokens, n_workers, max_tail_len):
        n = C.c_size_t()
        self.check(self.L.compact_prefix_stack_workspace_bytes(self.ctx, history_tokens, n_workers, max_tail_len, C.byref(n)))
        return n.value

    def compact_prefix_stack_forward(self, layer_weights, prefix_len, x_history, x_decode, shared, tails, y_decode):
        """layer_weights: one dict per layer; shared, tails: one KVCache per layer."""
        wsp, wsn = self._ws()
        nl = len(layer_weights)
        warr = (Weights * nl)()
        for l, wd in enumerate(layer_weights):
            for name, _ in Weights._fields_:
                t = wd.get(name)
                setattr(warr[l], name, t.data_ptr() if t is not None else None)
        sarr, tarr = (KV * nl)(), (KV * nl)()
        for l in range(nl):
            for name, _ in KV._fields_:
                setattr(sarr[l], name, getattr(shared[l].c, name))
                setattr(tarr[l], name, getattr(tails[l].c, name))
        S = 0 if x_decode is None else x_decode.shape[0]
        self.check(self.L.compact_prefix_stack_forward(
            self.ctx, nl, warr, tails[0].N, _i32arr(prefix_len), x_history.shape[0], _ptr(x_history), S, _ptr(x_decode),
            sarr, tarr, _ptr(y_decode), wsp, wsn, _stream()))

    # -- prefix-aware layout ------------------------------------------------------
    def prefix_workspace_bytes(self, n_workers, max_prefix_len, max_tail_len):
        n = C.c_size_t()
        self.check(self.L.compact_prefix_workspace_bytes(self.ctx, n_workers, max_prefix_len, max_tail_len, C.byref(n)))
        return n.value

    def compact_prefix_decode_step(self, x, shared, prefix_len, tails, y, route=None):
        wsp, wsn = self._ws()
        r = None if route is None else C.byref(RouteOut(route[0].data_ptr(), route[1].data_ptr()))
        self.check(self.L.compact_prefix_decode_step(self.ctx, C.byref(self.w), tails.N, _ptr(x), C.byref(shared.c),
                                                     _i32arr(prefix_len), C.byref(tails.c), _ptr(y), r, wsp, wsn, _stream()))

    def compact_attn_decode_prefix(self, q, shared, prefix_len, tails, o):
        wsp, wsn = self._ws()
        self.check(self.L.compact_attn_decode_prefix(self.ctx, tails.N, _ptr(q), C.byref(shared.c), _i32arr(prefix_len),
                                                     C.byref(tails.c), _ptr(o), wsp, wsn, _stream()))

    # -- paged cache in 8 bits ------------------------------------------------------
    # The kernels go by the sizes they are told, so every array is held against them here.  The comparisons are written out: with a
    # function call per array they cost 1.0 us a call instead of 0.7, of the 7 to 8 that a small one takes.
    def _fits(self, kv, device):
        if kv.heads != self.kv_heads or kv.device != device:
            _refuse("pages for %s KV heads x head_dim on device %d; the layer has %s, the current device is %d" % (kv.heads, kv.device, self.kv_heads, device))

    def compact_paged_plan(self, kv, step):
        device, ref, st = torch.cuda.current_device(), kv._ref or kv.struct(), step.struct()
        if step.n_requests != kv.n_requests or step.n_stack < kv.n_pages or step.head_dim != self.kv_heads[1] or kv.device != device or step.device != device:
            _refuse("step of %d requests, a stack of %d pages and head_dim %d on device %d; the cache has %d, %d, %d on device %d, the current device is %d"
                    % (step.n_requests, step.n_stack, step.head_dim, step.device, kv.n_requests, kv.n_pages, self.kv_heads[1], kv.device, device))
        rc = self.L.compact_paged_plan(self.ctx, ref, C.byref(st), _raw_stream(device))
        if rc:
            self.check(rc)

    def compact_rope_paged_write(self, qkv, kv, slot, rot, q):
        """qkv [rows, Dq + 2 Dkv] -> q [rows, Dq] (rotated), k and v into kv's pages at slot [rows]; rot [rows, hd / 2, 2].  slot, rot and
        q may have more rows."""
        device, ref, dt, shape = torch.cuda.current_device(), kv._ref or kv.struct(), self.torch_dtype, qkv.shape
        rows = shape[0]
        if (len(shape) != 2 or shape[1] != self.qkv_cols or kv.heads != self.kv_heads or kv.device != device
                or qkv.dtype is not dt or qkv.get_device() != device or not qkv.is_contiguous()
                or slot.dtype is not torch.int64 or slot.numel() < rows or slot.get_device() != device or not slot.is_contiguous()
                or rot.dtype is not torch.float32 or rot.numel() < rows * self.kv_heads[1] or rot.get_device() != device or not rot.is_contiguous()
                or q.dtype is not dt or q.numel() < rows * self.q_cols or q.get_device() != device or not q.is_contiguous()):
            self._fits(kv, device)
            _array(qkv, dt, 0, device, "qkv")
            _array(slot, torch.int64, rows, device, "slot")
            _array(rot, torch.float32, rows * self.kv_heads[1], device, "rot")
            _array(q, dt, rows * self.q_cols, device, "q")
            _refuse("qkv: %s, [rows, %d] needed" % (tuple(qkv.shape), self.qkv_cols))
        rc = self.L.compact_rope_paged_write(self.ctx, rows, qkv.data_ptr(), ref, slot.data_ptr(), rot.data_ptr(), q.data_ptr(), _raw_stream(device))
        if rc:
            self.check(rc)

    def paged_workspace_bytes(self, n_requests, n_rows, max_new, max_kv_len):
        n = C.c_size_t()
        self.check(self.L.compact_paged_workspace_bytes(self.ctx, n_requests, n_rows, max_new, max_kv_len, C.byref(n)))
        return n.value

    def ensure_paged_workspace(self, n_requests, n_rows, max_new, max_kv_len, device):
        need = self.paged_workspace_bytes(n_requests, n_rows, max_new, max_kv_len)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        return self.ws

    def compact_attn_paged(self, q, kv, cu, kv_len, max_new, max_kv_len, o):
        """q [rows, >= Dq] (its rows may be apart), o [rows, Dq], cu [n_requests + 1], kv_len [n_requests].  The workspace is self.ws."""
        device, ref, dt, shape, apart, ws = torch.cuda.current_device(), kv._ref or kv.struct(), self.torch_dtype, q.shape, q.stride(), self.ws
        rows, N = shape[0], kv.n_requests
        if (len(shape) != 2 or shape[1] < self.q_cols or apart[1] != 1 or kv.heads != self.kv_heads or kv.device != device
                or q.dtype is not dt or q.get_device() != device
                or cu.dtype is not torch.int32 or cu.numel() <= N or cu.get_device() != device or not cu.is_contiguous()
                or kv_len.dtype is not torch.int32 or kv_len.numel() < N or kv_len.get_device() != device or not kv_len.is_contiguous()
                or o.dtype is not dt or o.numel() < rows * self.q_cols or o.get_device() != device or not o.is_contiguous()
                or ws is not None and ws.get_device() != device):
            self._fits(kv, device)
            _array(cu, torch.int32, N + 1, device, "cu")
            _array(kv_len, torch.int32, N, device, "kv_len")
            _array(o, dt, rows * self.q_cols, device, "o")
            _refuse("q: %s %s with strides %s on %s, workspace on %s; [rows, %d] of %s on the current GPU needed"
                    % (q.dtype, tuple(q.shape), q.stride(), q.device, ws if ws is None else ws.device, self.q_cols, dt))
        rc = self.L.compact_attn_paged(self.ctx, ref, rows, cu.data_ptr(), kv_len.data_ptr(), max_new, max_kv_len, q.data_ptr(), apart[0],
                                       o.data_ptr(), None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _raw_stream(device))
        if rc:
            self.check(rc)

    # -- 8-bit integer weights ------------------------------------------------------
    # (every array is held against the sizes that the kernels go by; the comparisons are written out, as above)
    def compact_quant_i8(self, x, q, scale):
        """x [rows, cols] (its rows may be apart) -> codes q int8 [rows, cols], scale fp32 [rows]."""
        device, shape = torch.cuda.current_device(), x.shape
        if len(shape) != 2:
            _refuse("x: %s, [rows, cols] needed" % (tuple(shape),))
        rows, cols = shape
        apart, step = x.stride()
        if rows <= 1:
            apart = cols
        if (x.dtype is not self.torch_dtype or x.get_device() != device or step != 1 and cols > 1 or cols > MAX_INT
                or q.dtype is not torch.int8 or q.shape != shape or q.get_device() != device or not q.is_contiguous()
                or scale.dtype is not torch.float32 or scale.numel() < rows or scale.get_device() != device or not scale.is_contiguous()):
            _array(q, torch.int8, rows * cols, device, "codes")
            _array(scale, torch.float32, rows, device, "scale")
            _refuse("x: %s %s with strides %s on %s, codes %s; [rows, cols] of %s with whole rows on the current GPU, codes of its shape needed"
                    % (x.dtype, tuple(shape), x.stride(), x.device, tuple(q.shape), self.torch_dtype))
        rc = self.L.compact_quant_i8(self.ctx, x.data_ptr(), apart, rows, cols, q.data_ptr(), scale.data_ptr(), _raw_stream(device))
        if rc:
            self.check(rc)

    def gemm_i8_workspace_bytes(self, M, N, K, epilogue=0):
        n = C.c_size_t()
        self.check(self.L.compact_gemm_i8_workspace_bytes(self.ctx, M, N, K, epilogue, C.byref(n)))
        return n.value

    def compact_gemm_i8(self, a, a_scale, b, b_scale, r, c, epilogue=0):
        """a int8 [M, K], b int8 [N, K] (epilogue 1: [2N, K]), their scales fp32, r and c [M, N].  The workspace is self.ws, if there is one."""
        device, dt, ws = torch.cuda.current_device(), self.torch_dtype, self.ws
        if len(a.shape) != 2 or len(b.shape) != 2 or len(c.shape) != 2:
            _refuse("product: a %s, b %s, c %s; [M, K], [N, K] and [M, N] needed" % (tuple(a.shape), tuple(b.shape), tuple(c.shape)))
        (M, K), (M2, N), (n, K2) = a.shape, c.shape, b.shape
        if (M2 != M or K2 != K or n != (2 * N if epilogue == 1 else N) or N > MAX_INT or K > MAX_INT
                or a.dtype is not torch.int8 or a.get_device() != device or not a.is_contiguous()
                or b.dtype is not torch.int8 or b.get_device() != device or not b.is_contiguous()
                or a_scale.dtype is not torch.float32 or a_scale.numel() < M or a_scale.get_device() != device or not a_scale.is_contiguous()
                or b_scale.dtype is not torch.float32 or b_scale.numel() < n or b_scale.get_device() != device or not b_scale.is_contiguous()
                or c.dtype is not dt or c.get_device() != device or not c.is_contiguous()
                or r is not None and (r.dtype is not dt or r.shape != c.shape or r.get_device() != device or not r.is_contiguous())
                or ws is not None and ws.get_device() != device):
            _array(a, torch.int8, 0, device, "a")
            _array(b, torch.int8, 0, device, "b")
            _array(a_scale, torch.float32, M, device, "a_scale")
            _array(b_scale, torch.float32, n, device, "b_scale")
            _array(c, dt, 0, device, "c")
            if r is not None:
                _array(r, dt, 0, device, "r")
            _refuse("product: a %s, b %s, r %s, c %s, epilogue %d, workspace on %s do not belong together"
                    % (tuple(a.shape), tuple(b.shape), None if r is None else tuple(r.shape), tuple(c.shape), epilogue, None if ws is None else ws.device))
        rc = self.L.compact_gemm_i8(self.ctx, a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), None if r is None else r.data_ptr(),
                                    c.data_ptr(), M, N, K, epilogue, None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
                                    _raw_stream(device))
        if rc:
            self.check(rc)

    def compact_block_norm(self, x, b=None, g_post=None, gate=None, alpha=1.0, h=None, g_pre=None, n=None, q=None, q_scale=None):
        """Rows [rows, d_model]; h, n, q (int8) and q_scale (fp32 [rows]) are written where given.  gate: [d_model], or [rows, d_model] whose rows
        may be apart."""
        device, dt, shape, d = torch.cuda.current_device(), self.torch_dtype, x.shape, self.d_model
        rows = shape[0] if len(shape) == 2 else -1
        gate_stride = 0 if gate is None or rows <= 1 or gate.dim() == 1 else gate.stride(0)
        if (rows < 0 or shape[1] != d or x.dtype is not dt or x.get_device() != device or not x.is_contiguous()
                or b is not None and (b.dtype is not dt or b.shape != shape or b.get_device() != device or not b.is_contiguous())
                or h is not None and (h.dtype is not dt or h.shape != shape or h.get_device() != device or not h.is_contiguous())
                or n is not None and (n.dtype is not dt or n.shape != shape or n.get_device() != device or not n.is_contiguous())
                or g_post is not None and (g_post.dtype is not dt or g_post.numel() < d or g_post.get_device() != device or not g_post.is_contiguous())
                or g_pre is not None and (g_pre.dtype is not dt or g_pre.numel() < d or g_pre.get_device() != device or not g_pre.is_contiguous())
                or gate is not None and (gate.dtype is not dt or gate.get_device() != device or gate.shape != shape and tuple(gate.shape) != (d,)
                                         or gate.stride(-1) != 1)
                or q is not None and (q.dtype is not torch.int8 or q.shape != shape or q.get_device() != device or not q.is_contiguous())
                or q_scale is not None and (q_scale.dtype is not torch.float32 or q_scale.numel() < rows or q_scale.get_device() != device
                                            or not q_scale.is_contiguous())):
            if rows < 0 or shape[1] != d:
                _refuse("rows: %s, [rows, %d] needed" % (tuple(shape), d))
            for name, t, dtype, size in (("x", x, dt, rows * d), ("b", b, dt, rows * d), ("h", h, dt, rows * d), ("n", n, dt, rows * d), ("g_post", g_post, dt, d),
                                         ("g_pre", g_pre, dt, d), ("codes", q, torch.int8, rows * d), ("scale", q_scale, torch.float32, rows)):
                if t is not None:
                    _array(t, dtype, size, device, name)
            _refuse("rows %s: gate %s, b, h, n and codes %s; gate of %s [%d] or rows of it, the others of the rows' shape needed"
                    % (tuple(shape), None if gate is None else (gate.dtype, tuple(gate.shape), gate.stride()),
                       [None if t is None else tuple(t.shape) for t in (b, h, n, q)], dt, d))
        rc = self.L.compact_block_norm(self.ctx, x.data_ptr(), None if b is None else b.data_ptr(), None if g_post is None else g_post.data_ptr(),
                                       None if gate is None else gate.data_ptr(), gate_stride, alpha, None if h is None else h.data_ptr(),
                                       None if g_pre is None else g_pre.data_ptr(), None if n is None else n.data_ptr(),
                                       None if q is None else q.data_ptr(), None if q_scale is None else q_scale.data_ptr(), rows, _raw_stream(device))
        if rc:
            self.check(rc)

    def compact_route(self, rule, logits, bias, idx, weight, m=None, w_router=None):
        """logits fp32 [rows, n_experts], given, or written as m w_router^T where these are; bias fp32 [n_experts] or None; idx int32 and weight fp32
        [rows, top_k]."""
        device, (E, k), shape, f32 = torch.cuda.current_device(), self.experts, logits.shape, torch.float32
        rows = shape[0] if len(shape) == 2 else -1
        if (rows < 0 or shape[1] != E or logits.dtype is not f32 or logits.get_device() != device or not logits.is_contiguous()
                or bias is not None and (bias.dtype is not f32 or bias.numel() < E or bias.get_device() != device or not bias.is_contiguous())
                or idx.dtype is not torch.int32 or idx.numel() < rows * k or idx.get_device() != device or not idx.is_contiguous()
                or weight.dtype is not f32 or weight.numel() < rows * k or weight.get_device() != device or not weight.is_contiguous()
                or m is not None and m.shape != (rows, self.d_model) or w_router is not None and w_router.shape != (E, self.d_model)):
            if rows >= 0 and shape[1] == E:
                _array(logits, f32, 0, device, "logits")
                _array(idx, torch.int32, rows * k, device, "idx")
                _array(weight, f32, rows * k, device, "weight")
                if bias is not None:
                    _array(bias, f32, E, device, "bias")
            _refuse("router: logits %s, rows %s, weights %s; [rows, %d], [rows, %d] and [%d, %d] needed"
                    % (tuple(shape), None if m is None else tuple(m.shape), None if w_router is None else tuple(w_router.shape), E, self.d_model, E, self.d_model))
        rc = self.L.compact_route(self.ctx, rule.ref, None if m is None else _array(m, self.torch_dtype, 0, device, "rows"),
                                  None if w_router is None else _array(w_router, self.torch_dtype, 0, device, "router weights"), logits.data_ptr(),
                                  None if bias is None else bias.data_ptr(), rows, idx.data_ptr(), weight.data_ptr(), _raw_stream(device))
        if rc:
            self.check(rc)

    def moe_ffn_i8_workspace_bytes(self, rows):
        n = C.c_size_t()
        self.check(self.L.compact_moe_ffn_i8_workspace_bytes(self.ctx, rows, C.byref(n)))
        return n.value

    def compact_moe_ffn_i8(self, experts, m, m_scale, h, idx, weight, y):
        """experts: ExpertsI8; m int8 [rows, d], m_scale fp32 [rows], h and y [rows, d], idx int32 and weight fp32 [rows, top_k].  The workspace is
        self.ws."""
        device, dt, i8, f32, ws = torch.cuda.current_device(), self.torch_dtype, torch.int8, torch.float32, self.ws
        d, F, E, k, shape = self.layer.d_model, self.layer.ffn_dim, self.layer.n_experts, self.layer.top_k, m.shape
        if len(shape) != 2 or shape[1] != d or h.shape != shape or y.shape != shape or ws is not None and ws.get_device() != device:
            _refuse("rows: codes %s, h %s, y %s, workspace on %s; [rows, %d] on the current GPU needed"
                    % (tuple(shape), tuple(h.shape), tuple(y.shape), None if ws is None else ws.device, d))
        rows = shape[0]
        if experts.gate_up.shape != (E, 2 * F, d) or experts.down.shape != (E, d, F):
            _refuse("experts: gate_up %s, down %s; %s and %s needed" % (tuple(experts.gate_up.shape), tuple(experts.down.shape), (E, 2 * F, d), (E, d, F)))
        e = ExpertsI8Struct(_array(experts.gate_up, i8, 0, device, "gate_up"), _array(experts.gate_up_scale, f32, E * 2 * F, device, "gate_up_scale"),
                            _array(experts.down, i8, 0, device, "down"), _array(experts.down_scale, f32, E * d, device, "down_scale"))
        rc = self.L.compact_moe_ffn_i8(self.ctx, C.byref(e), _array(m, i8, 0, device, "codes"), _array(m_scale, f32, rows, device, "scale"),
                                       _array(h, dt, 0, device, "h"), _array(idx, torch.int32, rows * k, device, "idx"),
                                       _array(weight, f32, rows * k, device, "weight"), rows, _array(y, dt, 0, device, "y"),
                                       None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _raw_stream(device))
        if rc:
            self.check(rc)

    # -- profiling --------------------------------------------------------------
    def compact_profile_select(self, klass):
        self.check(self.L.compact_profile_select(self.ctx, klass))

    def compact_profile_read(self):
        n, ms = C.c_int64(), C.c_double()
        self.check(self.L.compact_profile_read(self.ctx, C.byref(n), C.byref(ms)))
        return n.value, ms.value

    # -- per-kernel entry points --------------------------------------------------
    def compact_mxfp4_dequant(self, codes, scales, out):
        """codes uint8 [..., K/2], scales uint8 [..., K/32] -> out bf16 [..., K]."""
        K = codes.shape[-1] * 2
        self.check(self.L.compact_mxfp4_dequant(self.ctx, _ptr(codes), _ptr(scales), codes.numel() // (K // 2), K, _ptr(out),
                                                _stream()))

    def compact_rmsnorm(self, x, g, y):
        self.check(self.L.compact_rmsnorm(self.ctx, _ptr(x), _ptr(g), _ptr(y), x.shape[0], _stream()))

    def compact_rope_kvwrite(self, cu_seqlens, qkv, kv):
        self.check(self.L.compact_rope_kvwrite(self.ctx, len(cu_seqlens) - 1, _i32arr(cu_seqlens), _ptr(qkv),
                                               C.byref(kv.c), _stream()))

    def compact_gemm(self, a, b, r, c, epilogue=0):
        wsp, wsn = self._ws()
        M, K = a.shape
        N = c.shape[1]
        self.check(self.L.compact_gemm(self.ctx, _ptr(a), _ptr(b), _ptr(r), _ptr(c), M, N, K, epilogue, wsp, wsn,
                                       _stream()))

    def compact_attn_prefill(self, cu_seqlens, qkv, kv, o):
        self.check(self.L.compact_attn_prefill(self.ctx, len(cu_seqlens) - 1, _i32arr(cu_seqlens), _ptr(qkv),
                                               C.byref(kv.c), _ptr(o), _stream()))

    def compact_attn_decode(self, q, kv, o):
        wsp, wsn = self._ws()
        self.check(self.L.compact_attn_decode(self.ctx, kv.N, _ptr(q), C.byref(kv.c), _ptr(o), wsp, wsn, _stream()))

    def compact_attn_decode_noalloc(self, q, kv, o):
        self.check(self.L.compact_attn_decode_noalloc(self.ctx, kv.N, _ptr(q), C.byref(kv.c), _ptr(o), _stream()))

    def compact_moe_route(self, m, w_router, idx, gate, logits=None):
        wsp, wsn = self._ws()
        self.check(self.L.compact_moe_route(self.ctx, _ptr(m), _ptr(w_router), m.shape[0], _ptr(idx), _ptr(gate),
                                            _ptr(logits), wsp, wsn, _stream()))

    def compact_moe_ffn(self, m, h, idx, gate, y):
        wsp, wsn = self._ws()
        self.check(self.L.compact_moe_ffn(self.ctx, C.byref(self.w), _ptr(m), _ptr(h), _ptr(idx), _ptr(gate),
                                          m.shape[0], _ptr(y), wsp, wsn, _stream()))
