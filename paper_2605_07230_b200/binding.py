"""Thin ctypes binding of libcascade.so (the C ABI declared in include/cascade.h).

Argument marshalling only: every step of the verification path runs inside the library's CUDA
kernels.  Tensors are torch tensors used as device (or pinned host) memory; their data pointers and
the current CUDA stream are passed straight through.  If the shared library is missing the import of
`lib()` raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcascade.so")

OK = 0
ERR_INVALID_ARG, ERR_BAD_TREE, ERR_WORKSPACE, ERR_UNSUPPORTED_SHAPE, ERR_CUDA, ERR_TIMEOUT = -1, -2, -3, -4, -5, -6
ERR_OVERFLOW, ERR_BAD_PAGE = -7, -8
F32, BF16 = 0, 1
USE_I, USE_C, CONV_DIST_SELF = 1, 2, 4
SELECT_LONGEST, SELECT_FIRST_ACCEPT = 0, 1
KERNEL_COUNT = 32
MAX_REQUESTS = 4096

EXPORTS = [
    "cascade_create", "cascade_destroy", "cascade_workspace_bytes", "cascade_check", "cascade_last_launch_count",
    "cascade_strerror", "cascade_timing_enable", "cascade_timing_read", "cascade_kernel_name", "cascade_tree_create", "cascade_tree_destroy", "cascade_tree_update", "cascade_tree_rows", "cascade_tree_depth",
    "cascade_tree_num_pairs", "cascade_tree_pairs", "cascade_tree_attn", "cascade_lm_head_cfg",
    "cascade_similarity", "cascade_relaxed_accept", "cascade_select_path", "cascade_verify_step",
    "cascade_verify_step_host", "cascade_accept_static", "cascade_bonus_token", "cascade_kv_append",
    "cascade_filter_logits", "cascade_set_wait_limit", "cascade_wait_probe",
    "cascade_tree_update_device", "cascade_tree_download", "cascade_drafter_loss",
    "cascade_paged_tables", "cascade_paged_append", "cascade_paged_attn", "cascade_sample",
]


class Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "B", "T_max", "P_max", "h", "Hq", "Hkv", "D", "V", "ffn")]


class Params(C.Structure):
    _fields_ = [("tau_pos", C.c_float), ("tau_seq", C.c_float), ("tvd_budget", C.c_float), ("flags", C.c_uint32)]


class Layer(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("gamma_attn", "wq", "wk", "wv", "wo", "gamma_mlp", "w_gate", "w_up",
                                          "w_down", "k_prefix", "v_prefix")]


class Step(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("layers", C.POINTER(Layer)), ("embed", C.c_void_p), ("gamma_final", C.c_void_p),
        ("w_head", C.c_void_p), ("prefix_cap", C.c_int32), ("prefix_len", C.c_void_p),
        ("eps", C.c_float), ("rope_base", C.c_float), ("softmax_scale", C.c_float), ("cfg_scale", C.c_float),
        ("temperature", C.c_float),
        ("tok", C.c_void_p), ("draft_p", C.c_void_p), ("uniforms", C.c_void_p), ("hidden_in", C.c_void_p),
        ("q", C.c_void_p), ("k_tree", C.c_void_p), ("v_tree", C.c_void_p), ("k_prefix", C.c_void_p),
        ("v_prefix", C.c_void_p), ("attn_out", C.c_void_p),
        ("params", Params), ("select_mode", C.c_int32),
        ("accept", C.c_void_p), ("path_nodes", C.c_void_p), ("path_len", C.c_void_p), ("q_relaxed", C.c_void_p),
        ("tvd_out", C.c_void_p), ("tvd_used", C.c_void_p), ("near_count", C.c_void_p),
        ("logits", C.c_void_p), ("feat", C.c_void_p), ("scores", C.c_void_p), ("row_lse", C.c_void_p),
        ("hidden_out", C.c_void_p), ("k_tree_out", C.c_void_p), ("v_tree_out", C.c_void_p),
        ("top_k", C.c_int32), ("top_p", C.c_float),
    ]


class PagedCacheStruct(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("page_stride", C.c_int64), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("block_table", C.c_void_p), ("table_stride", C.c_int32), ("table_width", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """Load libcascade.so (once).  Raises if it has not been built: there is no other code path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2605_07230_b200.build)")
        L = C.CDLL(LIB_PATH)
        L.cascade_strerror.restype = C.c_char_p
        L.cascade_workspace_bytes.restype = C.c_int64
        vp = C.c_void_p
        L.cascade_create.argtypes = [C.POINTER(vp), C.POINTER(Shape)]
        L.cascade_destroy.argtypes = [vp]
        L.cascade_workspace_bytes.argtypes = [vp]
        L.cascade_check.argtypes = [vp, vp]
        L.cascade_last_launch_count.argtypes = [vp]
        L.cascade_timing_enable.argtypes = [vp, C.c_int32]
        L.cascade_timing_read.argtypes = [vp, vp, vp]
        L.cascade_kernel_name.argtypes = [C.c_int32]
        L.cascade_kernel_name.restype = C.c_char_p
        L.cascade_tree_create.argtypes = [vp, C.c_int32, vp, C.POINTER(vp)]
        L.cascade_tree_destroy.argtypes = [vp]
        L.cascade_tree_update.argtypes = [vp, C.c_int32, vp, vp]
        for f in ("cascade_tree_rows", "cascade_tree_depth", "cascade_tree_num_pairs"):
            getattr(L, f).argtypes = [vp]
        L.cascade_tree_pairs.argtypes = [vp, vp, vp]
        L.cascade_tree_attn.argtypes = [vp, vp, vp, vp, vp, C.c_int32, vp, vp, vp, vp, C.c_float, vp]
        L.cascade_lm_head_cfg.argtypes = [vp, vp, vp, vp, C.c_float, vp, C.c_float, C.c_float, vp, vp, vp, vp, vp,
                                          vp, vp, vp]
        L.cascade_similarity.argtypes = [vp, vp, vp, C.c_int32, vp, vp, vp]
        L.cascade_relaxed_accept.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.POINTER(Params), vp, vp, vp,
                                             vp, vp]
        L.cascade_select_path.argtypes = [vp, vp, vp, vp, C.c_int32, vp, vp, vp, vp]
        L.cascade_verify_step.argtypes = [vp, vp, C.POINTER(Step), vp]
        L.cascade_verify_step_host.argtypes = [vp, vp, C.POINTER(Step), vp, vp, vp, vp, vp, vp, vp]
        L.cascade_accept_static.argtypes = [C.c_int32, C.c_int32, vp, vp, C.c_int32, vp, vp, vp, vp, vp, vp, vp,
                                            C.POINTER(Params), C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.cascade_bonus_token.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.cascade_kv_append.argtypes = [vp, vp, C.c_int32, C.POINTER(Layer), vp, vp, vp, vp, C.c_int32, vp, vp]
        L.cascade_filter_logits.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_float, vp, vp]
        L.cascade_tree_update_device.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, vp, vp]
        L.cascade_tree_download.argtypes = [vp, vp, vp, vp, vp, vp]
        L.cascade_drafter_loss.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_float, vp, vp, vp, vp]
        i32, i64, f32 = C.c_int32, C.c_int64, C.c_float
        cache = C.POINTER(PagedCacheStruct)
        L.cascade_paged_tables.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.cascade_paged_append.argtypes = [vp, cache, i32, vp, i64, vp, i64, vp, i64, vp, vp, f32, vp, i64, vp]
        L.cascade_paged_attn.argtypes = [vp, cache, i32, i32, vp, i64, vp, vp, i32, i32, i32, i32, f32, vp, vp, vp]
        L.cascade_sample.argtypes = [vp, vp, i32, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.cascade_set_wait_limit.argtypes = [vp, C.c_int64]
        L.cascade_wait_probe.argtypes = [vp, vp, vp]
        _lib = L
    return _lib


class CascadeError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"cascade status {status}: {lib().cascade_strerror(status).decode()}")


def _check(status: int) -> None:
    if status != OK:
        raise CascadeError(status)


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors must be contiguous"
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


class Context:
    """cascade_create / cascade_destroy."""

    def __init__(self, dtype: int, B: int, T_max: int, P_max: int, h: int, Hq: int, Hkv: int, D: int, V: int,
                 ffn: int = 0):
        self.shape = Shape(dtype, B, T_max, P_max, h, Hq, Hkv, D, V, ffn)
        self.handle = C.c_void_p()
        _check(lib().cascade_create(C.byref(self.handle), C.byref(self.shape)))

    def close(self):
        if self.handle:
            lib().cascade_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def workspace_bytes(self) -> int:
        return lib().cascade_workspace_bytes(self.handle)

    @property
    def last_launch_count(self) -> int:
        return lib().cascade_last_launch_count(self.handle)

    def check(self) -> None:
        _check(lib().cascade_check(self.handle, _stream()))

    def set_wait_limit(self, limit_ns: int) -> None:
        _check(lib().cascade_set_wait_limit(self.handle, int(limit_ns)))

    def wait_probe(self, waited_ns=None) -> None:
        """Enqueues the failure-path self-test (a wait that cannot end); check() raises ERR_TIMEOUT afterwards."""
        _check(lib().cascade_wait_probe(self.handle, _ptr(waited_ns), _stream()))

    def timing_enable(self, on: bool) -> None:
        _check(lib().cascade_timing_enable(self.handle, int(on)))

    def timing_read(self) -> dict:
        """{kernel name: (total ms, launches)} accumulated since the last read."""
        n = KERNEL_COUNT
        ms = (C.c_float * n)()
        cnt = (C.c_int32 * n)()
        _check(lib().cascade_timing_read(self.handle, ms, cnt))
        out = {}
        for i in range(n):
            name = lib().cascade_kernel_name(i)
            if name is not None and cnt[i] > 0:
                out[name.decode()] = (float(ms[i]), int(cnt[i]))
        return out


class Tree:
    """cascade_tree_create / cascade_tree_destroy.  `parent` is a host int32 sequence."""

    def __init__(self, ctx: Context, parent):
        self.ctx = ctx
        arr = (C.c_int32 * len(parent))(*[int(x) for x in parent])
        self.handle = C.c_void_p()
        _check(lib().cascade_tree_create(ctx.handle, len(parent), arr, C.byref(self.handle)))
        self.T = lib().cascade_tree_rows(self.handle)
        self.depth = lib().cascade_tree_depth(self.handle)
        self.num_pairs = lib().cascade_tree_num_pairs(self.handle)

    def update(self, parent):
        """A new tree in the same descriptor (no allocation); enqueued on the current stream."""
        arr = (C.c_int32 * len(parent))(*[int(x) for x in parent])
        _check(lib().cascade_tree_update(self.handle, len(parent), arr, _stream()))
        self.T = lib().cascade_tree_rows(self.handle)
        self.depth = lib().cascade_tree_depth(self.handle)
        self.num_pairs = lib().cascade_tree_num_pairs(self.handle)

    def update_device(self, T: int, depth_cap: int, pairs_cap: int, parent_dev):
        """A new tree from a device-resident int32 parent[] (no host round trip); enqueued on the current stream."""
        _check(lib().cascade_tree_update_device(self.handle, T, depth_cap, pairs_cap, _ptr(parent_dev), _stream()))
        self.T = lib().cascade_tree_rows(self.handle)
        self.depth = lib().cascade_tree_depth(self.handle)
        self.num_pairs = lib().cascade_tree_num_pairs(self.handle)

    def download(self):
        """The descriptor's device arrays as host lists: parent, depth, child_begin, child_count, anc (T x 4 words)."""
        T = self.T
        arrs = [(C.c_int32 * T)() for _ in range(4)]
        anc = (C.c_uint64 * (4 * T))()
        _check(lib().cascade_tree_download(self.handle, *arrs, anc))
        return [list(a) for a in arrs] + [[list(anc[4 * j: 4 * j + 4]) for j in range(T)]]

    def pairs(self):
        a = (C.c_int32 * max(self.num_pairs, 1))()
        b = (C.c_int32 * max(self.num_pairs, 1))()
        _check(lib().cascade_tree_pairs(self.handle, a, b))
        return list(a)[: self.num_pairs], list(b)[: self.num_pairs]

    def close(self):
        if self.handle:
            lib().cascade_tree_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def cascade_tree_attn(ctx, tree, q, k_prefix, v_prefix, prefix_cap, prefix_len, k_tree, v_tree, out, softmax_scale):
    _check(lib().cascade_tree_attn(ctx.handle, tree.handle, _ptr(q), _ptr(k_prefix), _ptr(v_prefix), prefix_cap,
                                   _ptr(prefix_len), _ptr(k_tree), _ptr(v_tree), _ptr(out), softmax_scale,
                                   _stream()))


def cascade_lm_head_cfg(ctx, tree, hidden, rms_gamma, eps, w_head, cfg_scale, temperature, tok, logits_out,
                        feat_out, feat_norm_out, row_lse_out, cand_parent_out, cand_gparent_out):
    _check(lib().cascade_lm_head_cfg(ctx.handle, tree.handle, _ptr(hidden), _ptr(rms_gamma), eps, _ptr(w_head),
                                     cfg_scale, temperature, _ptr(tok), _ptr(logits_out), _ptr(feat_out),
                                     _ptr(feat_norm_out), _ptr(row_lse_out), _ptr(cand_parent_out),
                                     _ptr(cand_gparent_out), _stream()))


def cascade_similarity(ctx, tree, feat, feat_dim, feat_norm, scores_out):
    _check(lib().cascade_similarity(ctx.handle, tree.handle, _ptr(feat), feat_dim, _ptr(feat_norm),
                                    _ptr(scores_out), _stream()))


def cascade_relaxed_accept(ctx, tree, scores, logits, row_lse, cand_parent, cand_gparent, tok, draft_p, uniforms,
                           params: Params, accept, q_relaxed, tvd_out, near_count):
    _check(lib().cascade_relaxed_accept(ctx.handle, tree.handle, _ptr(scores), _ptr(logits), _ptr(row_lse),
                                        _ptr(cand_parent), _ptr(cand_gparent), _ptr(tok), _ptr(draft_p),
                                        _ptr(uniforms), C.byref(params), _ptr(accept), _ptr(q_relaxed),
                                        _ptr(tvd_out), _ptr(near_count), _stream()))


def cascade_select_path(ctx, tree, accept, tvd_out, mode, path_nodes, path_len, tvd_used):
    _check(lib().cascade_select_path(ctx.handle, tree.handle, _ptr(accept), _ptr(tvd_out), mode, _ptr(path_nodes),
                                     _ptr(path_len), _ptr(tvd_used), _stream()))


def make_step(**kw) -> Step:
    """Fill a Step from keyword arguments; tensors become pointers, `layers` a list of dicts of tensors.
    The returned struct keeps references to everything it points to."""
    st = Step()
    keep = []
    layers = kw.pop("layers", None) or []
    st.n_layers = len(layers)
    if layers:
        arr = (Layer * len(layers))()
        for i, lw in enumerate(layers):
            for name, _ in Layer._fields_:
                setattr(arr[i], name, _ptr(lw[name]))
                keep.append(lw[name])
        st.layers = arr
        keep.append(arr)
    params = kw.pop("params")
    st.params = params
    for name, ctype in Step._fields_:
        if name in ("n_layers", "layers", "params"):
            continue
        if name not in kw:
            continue
        v = kw.pop(name)
        if ctype is C.c_void_p:
            setattr(st, name, _ptr(v))
            keep.append(v)
        else:
            setattr(st, name, v)
    assert not kw, f"unknown step fields: {sorted(kw)}"
    st._keep = keep
    return st


def cascade_verify_step(ctx, tree, step: Step):
    _check(lib().cascade_verify_step(ctx.handle, tree.handle, C.byref(step), _stream()))


def cascade_verify_step_host(ctx, tree, step: Step, tok_host, draft_p_host, uniforms_host, accept_host,
                             path_nodes_host, path_len_host):
    _check(lib().cascade_verify_step_host(ctx.handle, tree.handle, C.byref(step), _ptr(tok_host),
                                          _ptr(draft_p_host), _ptr(uniforms_host), _ptr(accept_host),
                                          _ptr(path_nodes_host), _ptr(path_len_host), _stream()))


def cascade_accept_static(B, parent, feat, feat_dim, feat_norm, row_lse, cand_parent, cand_gparent, tok, draft_p,
                          uniforms, params: Params, select_mode, accept, q_relaxed, tvd_out, near_count, path_nodes,
                          path_len, tvd_used):
    """Scores + relaxed acceptance + path selection with no context, no tree object and no device
    allocation (the library's static device array is the only scratch).  `parent` is a host sequence."""
    arr = (C.c_int32 * len(parent))(*[int(x) for x in parent])
    _check(lib().cascade_accept_static(B, len(parent), arr, _ptr(feat), feat_dim, _ptr(feat_norm), _ptr(row_lse),
                                       _ptr(cand_parent), _ptr(cand_gparent), _ptr(tok), _ptr(draft_p),
                                       _ptr(uniforms), C.byref(params), select_mode, _ptr(accept), _ptr(q_relaxed),
                                       _ptr(tvd_out), _ptr(near_count), _ptr(path_nodes), _ptr(path_len),
                                       _ptr(tvd_used), _stream()))


def cascade_filter_logits(ctx, logits, top_k, top_p, kept_count=None):
    n_rows = logits.numel() // logits.shape[-1]
    _check(lib().cascade_filter_logits(ctx.handle, _ptr(logits), n_rows, int(top_k), float(top_p), _ptr(kept_count),
                                       _stream()))


def cascade_bonus_token(ctx, tree, logits, tok, path_nodes, path_len, u_bonus, token_out, mass_out=None,
                        draft_row=None):
    _check(lib().cascade_bonus_token(ctx.handle, tree.handle, _ptr(logits), _ptr(tok), _ptr(draft_row),
                                     _ptr(path_nodes), _ptr(path_len), _ptr(u_bonus), _ptr(token_out),
                                     _ptr(mass_out), _stream()))


def cascade_kv_append(ctx, tree, step: Step, k_tree, v_tree, path_nodes, path_len, prefix_cap, prefix_len):
    """Appends the accepted path's rows to the caches named in `step.layers` (a Step made by make_step)."""
    _check(lib().cascade_kv_append(ctx.handle, tree.handle, step.n_layers, step.layers, _ptr(k_tree), _ptr(v_tree),
                                   _ptr(path_nodes), _ptr(path_len), prefix_cap, _ptr(prefix_len), _stream()))


def cascade_drafter_loss(target_logits, draft_logits, feat, tau_seq, c, loss_out, weight_out=None, total_out=None):
    """Eq. 4 of the paper on [K,V] target / drafter logits and [K,h] target hidden states (device tensors)."""
    K, V = target_logits.shape
    _check(lib().cascade_drafter_loss(_ptr(target_logits), _ptr(draft_logits), _ptr(feat), K, V, feat.shape[-1],
                                      float(tau_seq), float(c), _ptr(loss_out), _ptr(weight_out), _ptr(total_out),
                                      _stream()))


# ---- paged cache and sampling -----------------------------------------------------------------------------------------
# These calls sit in a decode loop where a launch lasts a few microseconds, so their checks stay short.


def _elem(ctx):
    return torch.bfloat16 if ctx.shape.dtype == BF16 else torch.float32


def _vector(name, t, dtype, n):
    """A dense tensor of n elements (None: not given); its address."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a dense {dtype} tensor of {n} elements, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _rows(name, t, n, heads, D, dtype):
    """Row stride of a [n,heads,D] tensor whose rows may lie apart (a part of a stacked projection)."""
    if t.dtype is not dtype or t.shape != (n, heads, D):
        raise ValueError(f"{name}: expected {dtype} {(n, heads, D)}, got {t.dtype} {tuple(t.shape)}")
    st = t.stride()
    if st[2] != 1 or (heads > 1 and st[1] != D):
        raise ValueError(f"{name}: heads and their elements must be dense, strides are {st}")
    return heads * D if n == 1 else st[0]


def _on_device(*tensors):
    """Every tensor given lives on the current device; its current stream."""
    dev = None
    for t in tensors:
        if t is not None:
            d = t.get_device()
            if d < 0 or (dev is not None and d != dev):
                raise ValueError(f"a tensor lives on {t.device}, not on the current CUDA device")
            dev = d
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"tensors live on cuda:{dev}, not on the current CUDA device")
    return torch._C._cuda_getCurrentRawStream(dev)


class PagedCache:
    """A cascade_paged_cache over [n_pages,page_size,Hkv,D] pools (pages may lie apart) and an int32 block table."""

    def __init__(self, k_pages, v_pages, block_table):
        if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype:
            raise ValueError("k_pages and v_pages must be [n_pages, page_size, Hkv, D] of one type and shape")
        n_pages, page, Hkv, D = k_pages.shape
        for t in (k_pages, v_pages):
            if t.stride(3) != 1 or (Hkv > 1 and t.stride(2) != D) or (page > 1 and t.stride(1) != Hkv * D):
                raise ValueError("the rows of a page must be dense")
        if n_pages > 1 and k_pages.stride(0) != v_pages.stride(0):
            raise ValueError("k_pages and v_pages must have the same page stride")
        if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.stride(1) != 1:
            raise ValueError("block_table must be int32 [n_req, width] with dense rows")
        self.k_pages, self.v_pages, self.block_table = k_pages, v_pages, block_table
        self.dtype, self.heads, self.n_req = k_pages.dtype, (Hkv, D), block_table.shape[0]
        stride = k_pages.stride(0) if n_pages > 1 else page * Hkv * D
        width = block_table.shape[1]                  # rows may lie further apart (columns of a wider table)
        row = width if self.n_req == 1 or width == 0 else block_table.stride(0)
        self.struct = PagedCacheStruct(k_pages.data_ptr(), v_pages.data_ptr(), stride, n_pages, page,
                                       block_table.data_ptr(), row, min(width, row))
        self.ref = C.byref(self.struct)

    def _check(self, ctx):
        sh = ctx.shape
        if self.dtype is not _elem(ctx) or self.heads != (sh.Hkv, sh.D):
            raise ValueError("the pool's element type, key heads or head size are not the context's")


def cascade_paged_tables(ctx, page_size, n_pages, new_len, kv_len, block_table, free_pages, free_count, kv_len_out,
                         free_count_out, q_begin, slot, pos):
    """Block tables, slot map and positions of the next pass; int32 device tensors (see include/cascade.h)."""
    n_req, n_tok, i32 = new_len.shape[0], slot.shape[0], torch.int32
    if block_table.dtype is not i32 or block_table.dim() != 2 or block_table.shape[0] != n_req or not block_table.is_contiguous():
        raise ValueError(f"block_table: expected a dense int32 tensor of {n_req} rows")
    new_p, kv_p, kv_out_p = (_vector("new_len", new_len, i32, n_req), _vector("kv_len", kv_len, i32, n_req),
                             _vector("kv_len_out", kv_len_out, i32, n_req))
    free_p, count_p, count_out_p = (_vector("free_pages", free_pages, i32, n_pages), _vector("free_count", free_count, i32, 1),
                                    _vector("free_count_out", free_count_out, i32, 1))
    begin_p, slot_p, pos_p = _vector("q_begin", q_begin, i32, n_req + 1), _vector("slot", slot, i32, n_tok), _vector("pos", pos, i32, n_tok)
    stream = _on_device(new_len, kv_len, block_table, free_pages, free_count, kv_len_out, free_count_out, q_begin, slot, pos)
    _check(lib().cascade_paged_tables(ctx.handle, n_req, n_tok, page_size, n_pages, new_p, kv_p, block_table.data_ptr(),
                                      block_table.shape[1], free_p, count_p, kv_out_p, count_out_p, begin_p, slot_p, pos_p, stream))


def cascade_paged_append(ctx, cache, k, v, slot, pos, rope_base=0.0, q=None, q_out=None):
    """Keys and values [n_tok,Hkv,D] (rotated unless rope_base is 0) into their slots; queries [n_tok,Hq,D] rotated."""
    cache._check(ctx)
    sh, e, n = ctx.shape, cache.dtype, slot.shape[0]
    Hkv, Hq, D = sh.Hkv, sh.Hq, sh.D
    slot_p, pos_p = _vector("slot", slot, torch.int32, n), _vector("pos", pos, torch.int32, n)
    ks, vs = _rows("k", k, n, Hkv, D, e), _rows("v", v, n, Hkv, D, e)
    q_p = q_out_p = None
    qs = qos = 0
    if q is not None:
        qs, q_p = _rows("q", q, n, Hq, D, e), q.data_ptr()
    if q_out is not None:
        qos, q_out_p = _rows("q_out", q_out, n, Hq, D, e), q_out.data_ptr()
    stream = _on_device(cache.k_pages, cache.v_pages, k, v, slot, pos, q, q_out)
    _check(lib().cascade_paged_append(ctx.handle, cache.ref, n, q_p, qs, k.data_ptr(), ks, v.data_ptr(), vs, slot_p, pos_p, rope_base,
                                      q_out_p, qos, stream))


def cascade_paged_attn(ctx, cache, q, q_begin, kv_len, max_q, max_kv, out, softmax_scale, window=0, sinks=0, lse=None):
    """Causal attention of each request's new tokens over its pages, optionally through a window beside sink tokens."""
    cache._check(ctx)
    sh, e, n_req, n = ctx.shape, cache.dtype, kv_len.shape[0], q.shape[0]
    Hq, D = sh.Hq, sh.D
    begin_p, kv_p = _vector("q_begin", q_begin, torch.int32, n_req + 1), _vector("kv_len", kv_len, torch.int32, n_req)
    if cache.n_req < n_req:
        raise ValueError(f"block_table has {cache.n_req} rows for {n_req} requests")
    qs = _rows("q", q, n, Hq, D, e)
    if out.dtype is not e or out.shape != (n, Hq, D) or not out.is_contiguous():
        raise ValueError(f"out: expected a dense {e} tensor of {(n, Hq, D)}")
    lse_p = None
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.shape != (n, Hq) or not lse.is_contiguous():
            raise ValueError(f"lse: expected a dense float32 tensor of {(n, Hq)}")
        lse_p = lse.data_ptr()
    stream = _on_device(cache.k_pages, cache.v_pages, cache.block_table, q, q_begin, kv_len, out, lse)
    _check(lib().cascade_paged_attn(ctx.handle, cache.ref, n_req, n, q.data_ptr(), qs, begin_p, kv_p, max_q, max_kv, window, sinks,
                                    softmax_scale, out.data_ptr(), lse_p, stream))


def cascade_sample(ctx, logits, uniforms, token, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, kept=None):
    """One token per row of [n_rows,V] float or bf16 logits (rows may lie apart); settings are device tensors per row."""
    dt, f32, i32 = logits.dtype, torch.float32, torch.int32
    if logits.dim() != 2 or logits.shape[1] != ctx.shape.V or (dt is not f32 and dt is not torch.bfloat16):
        raise ValueError(f"logits: expected float32 or bfloat16 [n_rows, {ctx.shape.V}], got {dt} {tuple(logits.shape)}")
    n, V = logits.shape
    st = logits.stride()
    if st[1] != 1:
        raise ValueError("a row of logits must be dense")
    args = (_vector("temperature", temperature, f32, n), _vector("top_k", top_k, i32, n), _vector("top_p", top_p, f32, n),
            _vector("min_p", min_p, f32, n), _vector("uniforms", uniforms, f32, n), _vector("token", token, i32, n),
            _vector("prob", prob, f32, n), _vector("kept", kept, i32, n))
    stream = _on_device(logits, uniforms, token, temperature, top_k, top_p, min_p, prob, kept)
    _check(lib().cascade_sample(ctx.handle, logits.data_ptr(), F32 if dt is f32 else BF16, V if n == 1 else st[0], n, *args, stream))
