"""MI355X (gfx950) group-batched step of JoyNexus multi-tenant group batching.

Thin Python binding of ``libjoynexus.so`` (C ABI in ``include/joynexus.h``):
the functions below carry the C names and only marshal arguments -- every
step of the path runs in the library's HIP kernels.  PyTorch supplies device
memory and streams.  Importing this package fails if the library is not
built; there is no fallback implementation.
"""
from __future__ import annotations

import ctypes as C
from typing import List, Optional, Sequence

import numpy as np

from . import _abi
from ._abi import (EXPERT_LAYER_FIELDS, JN_OK, STATUS_NAMES, jn_adamw_tenant, jn_backbone, jn_expert, jn_expert_io,
                   jn_expert_layer, jn_expert_layer_grads, jn_head, jn_head_io, jn_layer, jn_pack_opts,
                   jn_kv_attn, jn_kv_batch, jn_kv_cache, jn_pack_sizes, jn_packed, jn_qk_args, jn_request, jn_tenant,
                   jn_token_head, jn_token_io, jn_token_pick, jn_token_verify)

_lib = _abi.load()

__all__ = [
    "JNError", "Context", "Request", "Tenant", "Backbone", "Head", "HeadIO",
    "jn_pack_plan", "jn_pack_maps_host", "jn_pack_group", "jn_backbone_workspace_size",
    "jn_backbone_forward", "jn_heads_workspace_size", "jn_tenant_heads_fwd_bwd", "jn_tenant_heads_fwd_bwd_noalloc",
    "HEADS_SCRATCH_BYTES", "jn_unpack",
    "Expert", "ExpertIO", "jn_pack_tenant_sizes", "jn_experts_workspace_size", "jn_tenant_experts_fwd_bwd",
    "QKNormRope", "jn_qk_norm_rope", "jn_qk_norm_rope_workspace_size", "jn_qk_norm_rope_bwd",
    "KVCache", "KVBatch", "jn_kv_append", "jn_kv_attention_workspace_size", "jn_kv_attention", "jn_kv_keep",
    "jn_backbone_extend_workspace_size", "jn_backbone_extend",
    "TokenVerify", "jn_tokens_verify_workspace_size", "jn_tenant_tokens_verify",
    "TokenHead", "TokenIO", "TokenPick", "jn_tokens_workspace_size", "jn_tenant_tokens_fwd_bwd",
    "jn_tokens_decode_workspace_size", "jn_tenant_tokens_decode",
    "AdamWTenant", "jn_adamw_workspace_size", "jn_tenant_adamw_step",
    "Collector", "InferPlan", "jn_infer_workspace_size",
    "lib_path",
]


def lib_path() -> str:
    return _abi.LIB_PATH


class JNError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _check(st: int, ctx: "Context" = None, what: str = ""):
    if st != JN_OK:
        msg = _lib.jn_last_error(ctx.handle).decode() if ctx is not None else what
        raise JNError(st, msg or what)


_torch = None


def _dtypes():
    """torch, imported at its first use."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _ptr(t) -> int:
    """Device pointer of a torch tensor (or an int)."""
    if t is None:
        return None
    return t if isinstance(t, int) else t.data_ptr()


class Context:
    """A library context bound to a HIP stream (default: torch's current stream)."""

    def __init__(self, stream=None):
        import torch
        if stream is None:
            stream = torch.cuda.current_stream()
        self.stream = stream
        h = C.c_void_p()
        _check(_lib.jn_ctx_create(C.byref(h), C.c_void_p(stream.cuda_stream)), what="jn_ctx_create")
        self.handle = h

    def set_trace(self, enable: bool):
        """Bracket every kernel this context launches with timing events."""
        _check(_lib.jn_ctx_set_trace(self.handle, 1 if enable else 0), self)

    def set_option(self, option: int, value: int):
        """jn_ctx_set_option: e.g. ``_abi.JN_OPT_EXPERT_TRANSPOSES``."""
        _check(_lib.jn_ctx_set_option(self.handle, int(option), int(value)), self)

    def trace_read(self, cap: int = 1 << 16) -> list:
        """[(op name, M, N, K, ms)] of the traced launches, in launch order."""
        buf = (_abi.jn_trace_entry * cap)()
        n = C.c_int32()
        _check(_lib.jn_ctx_trace_read(self.handle, buf, cap, C.byref(n)), self)
        return [(_abi.OPS.get(e.op, str(e.op)), e.M, e.N, e.K, e.ms) for e in buf[: n.value]]

    def close(self):
        if self.handle:
            _lib.jn_ctx_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- marshal ---

class Request:
    """A tenant request: ``embeds`` device bf16 [n, max_len, d], host lengths."""

    def __init__(self, tenant: int, embeds, lengths, max_len: int = None):
        self.tenant = int(tenant)
        self.embeds = embeds
        self.lengths = np.ascontiguousarray(lengths, dtype=np.int32)
        self.n = int(self.lengths.shape[0])
        self.max_len = int(max_len) if max_len is not None else int(embeds.shape[1])


class Tenant:
    def __init__(self, prefix_sig: int, d_model: int):
        self.prefix_sig = int(prefix_sig)
        self.d_model = int(d_model)


def _requests(reqs: Sequence[Request]):
    arr = (jn_request * len(reqs))()
    keep = []
    for i, r in enumerate(reqs):
        lens = r.lengths
        keep.append(lens)
        arr[i].tenant = r.tenant
        arr[i].n_samples = r.n
        arr[i].max_len = r.max_len
        arr[i].embeds = _ptr(r.embeds) if r.embeds is not None else None
        arr[i].lengths = lens.ctypes.data_as(C.POINTER(C.c_int32))
    return arr, keep


def _tenants(ten: Sequence[Tenant]):
    arr = (jn_tenant * len(ten))()
    for i, t in enumerate(ten):
        arr[i].prefix_sig = t.prefix_sig
        arr[i].d_model = t.d_model
    return arr


def _opts(d: int, align: int):
    o = jn_pack_opts()
    o.d_model = d
    o.align = align
    return o


# ---------------------------------------------------------------- pack ------

def jn_pack_plan(reqs: Sequence[Request], tenants: Sequence[Tenant], d: int, align: int = 1) -> jn_pack_sizes:
    ra, keep = _requests(reqs)
    ta = _tenants(tenants)
    out = jn_pack_sizes()
    o = _opts(d, align)
    _check(_lib.jn_pack_plan(ra, len(reqs), ta, len(tenants), C.byref(o), C.byref(out)), what="jn_pack_plan")
    return out


def jn_pack_maps_host(reqs: Sequence[Request], tenants: Sequence[Tenant], d: int, align: int = 1) -> dict:
    """Index maps computed on the host by the library (numpy int32 arrays)."""
    sz = jn_pack_plan(reqs, tenants, d, align)
    buf = np.zeros(int(sz.map_bytes), dtype=np.uint8)
    ra, keep = _requests(reqs)
    ta = _tenants(tenants)
    out = jn_packed()
    o = _opts(d, align)
    _check(_lib.jn_pack_maps_host(ra, len(reqs), ta, len(tenants), C.byref(o),
                                  buf.ctypes.data_as(C.c_void_p), buf.nbytes, C.byref(out)), what="jn_pack_maps_host")
    base = buf.ctypes.data
    res = {"N": out.N, "T": out.T, "max_seqlen": out.max_seqlen, "req_sig": out.req_sig}
    for name in jn_packed.MAP_FIELDS:
        off = C.cast(getattr(out, name), C.c_void_p).value - base
        res[name] = buf[off: off + 4 * out.map_len(name)].view(np.int32).copy()
    return res


class Packed:
    """A packed batch: the C struct plus the tensors it points into."""

    def __init__(self, struct: jn_packed, maps, tokens):
        self.struct = struct
        self.maps = maps
        self.tokens = tokens

    def __getattr__(self, k):
        return getattr(self.struct, k)

    def map_tensor(self, name: str):
        """View of one device index map as an int32 tensor."""
        import torch
        off = C.cast(getattr(self.struct, name), C.c_void_p).value - self.maps.data_ptr()
        n = self.struct.map_len(name)
        return self.maps[off: off + 4 * n].view(torch.int32)


def jn_pack_group(ctx: Context, reqs: Sequence[Request], tenants: Sequence[Tenant], d: int, align: int,
                  maps, tokens) -> Packed:
    ra, keep = _requests(reqs)
    ta = _tenants(tenants)
    out = jn_packed()
    o = _opts(d, align)
    _check(_lib.jn_pack_group(ctx.handle, ra, len(reqs), ta, len(tenants), C.byref(o), _ptr(maps),
                              maps.numel() * maps.element_size(), _ptr(tokens),
                              tokens.numel() * tokens.element_size(), C.byref(out)), ctx)
    return Packed(out, maps, tokens)


# ------------------------------------------------------------ backbone ------

def _rope_fields(s, theta: float, sections, interleaved: bool):
    sections = [int(x) for x in sections or ()]
    if len(sections) > 4:
        raise ValueError("at most four position axes")
    s.rope_theta = float(theta)
    s.rope_axes = len(sections)
    s.rope_interleaved = 1 if interleaved else 0
    s.rope_sections = (C.c_int32 * 4)(*(sections + [0] * (4 - len(sections))))


def _positions(pos, rows: int, axes: int):
    """Device pointer of int32 positions [rows, axes] ([rows] with one axis)."""
    if pos is None:
        return None
    if pos.dtype is not _dtypes().int32 or not pos.is_contiguous() or pos.numel() != rows * axes:
        raise TypeError(f"positions must be a contiguous int32 tensor of {rows} x {axes}")
    return pos.data_ptr()


class Backbone:
    """Device weights of the frozen backbone (lists of torch bf16 tensors).

    A layer with head norms also has "gq" and "gk" (bf16 [head width]).  ``rope_sections``: pairs of every position
    axis, for rows with several positions.  Positions belong to a batch: the calls take them as ``pos``, and nothing
    here writes those of ``set_positions``, which stand for calls that give none."""

    def __init__(self, layers: List[dict], gf, n_heads: int, eps: float, n_kv_heads: int = 0, causal: bool = False,
                 rope_theta: float = 0.0, rope_sections: Sequence[int] = (), rope_interleaved: bool = False):
        self.layers = layers
        self.gf = gf
        self.n_heads = int(n_heads)
        self.n_kv_heads = int(n_kv_heads)
        self.causal = bool(causal)
        self.rope_theta = float(rope_theta)
        self.eps = float(eps)
        self.d = int(gf.shape[0])
        self.ffn = int(layers[0]["w_up"].shape[0])
        arr = (jn_layer * len(layers))()
        for i, L in enumerate(layers):
            arr[i].wqkv = _ptr(L["wqkv"])
            arr[i].wo = _ptr(L["wo"])
            arr[i].w_up = _ptr(L["w_up"])
            arr[i].w_gate = _ptr(L.get("w_gate"))
            arr[i].w_down = _ptr(L["w_down"])
            arr[i].g1 = _ptr(L["g1"])
            arr[i].g2 = _ptr(L["g2"])
            arr[i].gq = _ptr(L.get("gq"))
            arr[i].gk = _ptr(L.get("gk"))
        self._arr = arr
        s = jn_backbone()
        s.n_layers = len(layers)
        s.d = self.d
        s.n_heads = self.n_heads
        s.ffn = self.ffn
        s.eps = self.eps
        s.n_kv_heads = self.n_kv_heads
        s.causal = 1 if self.causal else 0
        _rope_fields(s, rope_theta, rope_sections, rope_interleaved)
        s.layers = C.cast(arr, C.POINTER(jn_layer))
        s.gf = _ptr(gf)
        self.struct = s
        self.pos = None

    def set_positions(self, pos):
        """Positions of the packed rows of calls that give none: device int32 [T, axes] (None: the rows' own)."""
        if pos is not None and pos.dim() != 2:
            raise TypeError("positions must be [T, axes]")
        self.struct.pos = _positions(pos, pos.shape[0] if pos is not None else 0, max(1, self.struct.rope_axes))
        self.pos = pos


def jn_backbone_workspace_size(bb: Backbone, T: int) -> int:
    n = C.c_size_t()
    _check(_lib.jn_backbone_workspace_size(C.byref(bb.struct), T, C.byref(n)), what="jn_backbone_workspace_size")
    return int(n.value)


def _backbone_of(bb: Backbone, T: int, pos):
    """The C struct for a batch of T rows at ``pos``, a copy where that is not the backbone's own."""
    own = getattr(bb, "pos", None)  # (anything with a `struct` may stand for a backbone)
    if pos is None:
        if own is not None and own.shape[0] != T:
            raise ValueError(f"the backbone's positions are of {own.shape[0]} rows, the batch has {T}")
        return bb.struct
    if pos.dim() != 2 or pos.shape[0] != T:
        raise ValueError(f"positions must be [{T}, axes], not {tuple(pos.shape)}")
    s = jn_backbone.from_buffer_copy(bb.struct)
    s.pos = _positions(pos, T, max(1, s.rope_axes))
    return s


def jn_backbone_forward(ctx: Context, bb: Backbone, packed: Packed, hidden, ws, pos=None):
    """``pos``: device int32 [T, axes], positions of the batch's packed rows (None: as ``Backbone.set_positions`` says)."""
    _check(_lib.jn_backbone_forward(ctx.handle, C.byref(_backbone_of(bb, packed.struct.T, pos)), C.byref(packed.struct),
                                    _ptr(hidden), _ptr(ws), ws.numel() * ws.element_size()), ctx)


# --------------------------------------- queries and keys: norm, rotation ---

class QKNormRope:
    """Head norms (``gq``, ``gk``: device bf16 [head_dim], or both None) and rotation (``theta`` > 0) of the query and
    key heads of fused rows; ``sections``: pairs of every position axis, none for a single axis."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, eps: float = 1e-6, gq=None, gk=None,
                 theta: float = 0.0, sections: Sequence[int] = (), interleaved: bool = False):
        self.gq, self.gk = gq, gk
        s = jn_qk_args()
        s.n_heads, s.n_kv_heads, s.head_dim = int(n_heads), int(n_kv_heads), int(head_dim)
        s.eps = float(eps)
        s.gq, s.gk = _ptr(gq), _ptr(gk)
        _rope_fields(s, theta, sections, interleaved)
        self.struct = s

        self.axes = max(1, s.rope_axes)
        self.width = (s.n_heads + s.n_kv_heads) * s.head_dim

    def at(self, rows: int, pos, x=None, y=None, dx=None):
        """The C arguments for rows of x, y (or its gradient) and dx."""
        s = jn_qk_args.from_buffer_copy(self.struct)
        s.rows = rows
        s.pos = _positions(pos, rows, self.axes)
        if x is not None:
            s.ld_in = _row_stride(x, rows, self.width)
        if y is not None:
            s.ld_out = _row_stride(y, rows, self.width)
        if dx is not None:
            s.ld_grad = _row_stride(dx, rows, self.width)
        return s


def _row_stride(t, rows: int, width: int) -> int:
    """Elements between the rows of a bf16 [rows, >= width] tensor."""
    shape = t.shape
    if t.dtype is not _dtypes().bfloat16 or len(shape) != 2 or shape[0] != rows or shape[1] < width:
        raise TypeError(f"rows must be a bfloat16 tensor [{rows}, >= {width}]")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise TypeError("the columns of a row must be adjacent")
    return ld if rows > 1 else (max(ld, shape[1]) + 7) // 8 * 8  # (of one row any: nothing is that far away)


def jn_qk_norm_rope(ctx: Context, qk: QKNormRope, x, pos, y):
    a = qk.at(x.shape[0], pos, x, y)
    _check(_lib.jn_qk_norm_rope(ctx.handle, a, x.data_ptr(), y.data_ptr()), ctx)


def jn_qk_norm_rope_workspace_size(qk: QKNormRope, rows: int) -> int:
    n = C.c_size_t()
    a = jn_qk_args.from_buffer_copy(qk.struct)
    a.rows = int(rows)
    _check(_lib.jn_qk_norm_rope_workspace_size(C.byref(a), C.byref(n)), what="jn_qk_norm_rope_workspace_size")
    return int(n.value)


def _gain(t, qk: QKNormRope):
    if t is None:
        return None
    if t.dtype is not _dtypes().float32 or t.numel() != qk.struct.head_dim or not t.is_contiguous():
        raise TypeError("gain gradients must be contiguous float32 tensors [head_dim]")
    return t.data_ptr()


def _bytes(ws) -> int:
    return ws.numel() * ws.element_size() if ws is not None else 0


def jn_qk_norm_rope_bwd(ctx: Context, qk: QKNormRope, x, pos, dy, dx, dgq, dgk, ws):
    """``x``, ``dgq``, ``dgk`` and ``ws`` may be None without norms."""
    a = qk.at(dy.shape[0], pos, x, dy, dx)
    _check(_lib.jn_qk_norm_rope_bwd(ctx.handle, a, _ptr(x), dy.data_ptr(), dx.data_ptr(), _gain(dgq, qk), _gain(dgk, qk),
                                    _ptr(ws), _bytes(ws)), ctx)


# ----------------------------------------- keys and values of earlier rows ---

def _entries(name: str, t, dtype, n: int):
    if t is None or t.dtype is not dtype or not t.is_contiguous() or t.numel() != n:
        raise TypeError(f"{name} must be a contiguous {dtype} tensor of {n} elements")
    return t.data_ptr()


class KVCache:
    """A paged cache: device bf16 ``k`` and ``v`` [layers, pages, key heads, page size, head width], of equal strides,
    where heads, rows and elements of a page lie together."""

    def __init__(self, k, v):
        t = _dtypes()
        if k.dtype is not t.bfloat16 or v.dtype is not t.bfloat16 or k.dim() != 5 or v.shape != k.shape:
            raise TypeError("k and v must be bfloat16 tensors [layers, pages, heads, page size, head width]")
        layers, pages, kv, size, hd = k.shape
        ld_layer, ld_page, *inner = k.stride()
        if inner != [size * hd, hd, 1] or v.stride() != k.stride():
            raise TypeError("a page's heads and rows must lie together, in both caches alike")
        self.k, self.v = k, v
        s = jn_kv_cache()
        s.n_layers, s.n_pages, s.page_size, s.n_kv_heads, s.head_dim = layers, pages, size, kv, hd
        s.ld_page = ld_page if pages > 1 else kv * size * hd  # (of one page any distance: nothing is that far away)
        s.ld_layer = ld_layer
        s.k, s.v = k.data_ptr(), v.data_ptr()
        self.struct = s


class KVBatch:
    """New rows of cached sequences, all device int32: ``pages`` [sequences, pages of each], ``past`` (cached rows) and
    ``cu_rows`` [sequences + 1]; ``rows`` of a call, at most ``max_new`` of a sequence.  ``parents`` [rows]: trees (indices in
    the sequence's new rows); ``whole``: its new rows all see each other."""

    def __init__(self, pages, past, cu_rows, rows: int, max_new: int, parents=None, whole: bool = False):
        t = _dtypes()
        if pages.dim() != 2:
            raise TypeError("pages must be [sequences, pages of each]")
        n, per = pages.shape
        self.pages, self.past, self.cu_rows, self.parents = pages, past, cu_rows, parents
        s = jn_kv_batch()
        s.n_seqs, s.max_pages, s.rows, s.max_new, s.whole = int(n), int(per), int(rows), int(max_new), 1 if whole else 0
        s.pages = _entries("pages", pages, t.int32, n * per)
        s.past = _entries("past", past, t.int32, n)
        s.cu_rows = _entries("cu_rows", cu_rows, t.int32, n + 1)
        s.parents = _entries("parents", parents, t.int32, s.rows) if parents is not None else None
        self.struct = s


def jn_kv_append(ctx: Context, cache: KVCache, layer: int, batch: KVBatch, qk: QKNormRope, x, pos, q):
    """Rows of ``x`` (query, key and value heads): norms and rotation as ``qk`` says, keys and values to the cache,
    queries to ``q`` (``x`` itself, another, or None without query heads).  ``pos`` None: the rows' own places."""
    rows, s = batch.struct.rows, qk.struct
    a = jn_qk_args.from_buffer_copy(s)
    a.rows = rows
    a.pos = _positions(pos, rows, qk.axes)
    a.ld_in = _row_stride(x, rows, qk.width + s.n_kv_heads * s.head_dim)
    if q is not None:
        a.ld_out = _row_stride(q, rows, s.n_heads * s.head_dim)
    _check(_lib.jn_kv_append(ctx.handle, C.byref(cache.struct), layer, C.byref(batch.struct), a, x.data_ptr(), _ptr(q)), ctx)


def _kv_attn(cache: KVCache, n_heads: int, scale: float):
    a = jn_kv_attn()
    a.n_heads, a.scale = int(n_heads), float(scale)
    a.ld_q = a.ld_out = a.n_heads * cache.struct.head_dim
    return a


def jn_kv_attention_workspace_size(cache: KVCache, batch: KVBatch, n_heads: int) -> int:
    n = C.c_size_t()
    _check(_lib.jn_kv_attention_workspace_size(C.byref(cache.struct), C.byref(batch.struct), _kv_attn(cache, n_heads, 0.0),
                                               C.byref(n)), what="jn_kv_attention_workspace_size")
    return int(n.value)


def jn_kv_attention(ctx: Context, cache: KVCache, layer: int, batch: KVBatch, n_heads: int, q, out, ws, scale: float = 0.0):
    """``q`` and ``out``: bf16 [rows, >= n_heads x head width]; ``scale`` 0: 1 / sqrt(head width)."""
    a, rows = _kv_attn(cache, n_heads, scale), batch.struct.rows
    a.ld_q, a.ld_out = _row_stride(q, rows, a.ld_q), _row_stride(out, rows, a.ld_out)
    _check(_lib.jn_kv_attention(ctx.handle, C.byref(cache.struct), layer, C.byref(batch.struct), a, q.data_ptr(),
                                out.data_ptr(), _ptr(ws), _bytes(ws)), ctx)


def jn_kv_keep(ctx: Context, cache: KVCache, batch: KVBatch, path, n_path, past_out=None):
    """``path`` int32 [sequences, most rows], ``n_path`` [sequences]; ``past_out`` [sequences]: the new ``past``."""
    t, n = _dtypes(), batch.struct.n_seqs
    if path.dim() != 2:
        raise TypeError("path must be [sequences, most rows]")
    most = int(path.shape[1])
    _check(_lib.jn_kv_keep(ctx.handle, C.byref(cache.struct), C.byref(batch.struct), _entries("path", path, t.int32, n * most),
                           most, _entries("n_path", n_path, t.int32, n),
                           _entries("past_out", past_out, t.int32, n) if past_out is not None else None), ctx)


def jn_backbone_extend_workspace_size(bb: Backbone, cache: KVCache, batch: KVBatch, pos=None) -> int:
    n = C.c_size_t()
    _check(_lib.jn_backbone_extend_workspace_size(C.byref(_backbone_of(bb, batch.struct.rows, pos)), C.byref(cache.struct),
                                                  C.byref(batch.struct), C.byref(n)), what="jn_backbone_extend_workspace_size")
    return int(n.value)


def jn_backbone_extend(ctx: Context, bb: Backbone, cache: KVCache, batch: KVBatch, embeds, hidden, ws, pos=None):
    """``embeds`` and ``hidden``: contiguous bf16 [rows, d]; ``pos`` as in ``jn_backbone_forward``."""
    t, rows = _dtypes(), batch.struct.rows
    _check(_lib.jn_backbone_extend(ctx.handle, C.byref(_backbone_of(bb, rows, pos)), C.byref(cache.struct),
                                   C.byref(batch.struct), _entries("embeds", embeds, t.bfloat16, rows * bb.d),
                                   _entries("hidden", hidden, t.bfloat16, rows * bb.d), _ptr(ws), _bytes(ws)), ctx)


# --------------------------------------------------------------- heads ------

class Head:
    """A tenant's MLP head: lists of device fp32 W [out, in] and b [out]."""

    def __init__(self, W: list, b: list, action_dim: int, chunk: int):
        self.W, self.b = W, b
        self.dims = np.array([int(W[0].shape[1])] + [int(w.shape[0]) for w in W], dtype=np.int32)
        s = jn_head()
        s.n_layers = len(W)
        s.action_dim = int(action_dim)
        s.chunk = int(chunk)
        self._W = (C.c_void_p * len(W))(*[_ptr(w) for w in W])
        self._b = (C.c_void_p * len(b))(*[_ptr(x) for x in b])
        s.dims = self.dims.ctypes.data_as(C.POINTER(C.c_int32))
        s.W = C.cast(self._W, C.POINTER(C.c_void_p))
        s.b = C.cast(self._b, C.POINTER(C.c_void_p))
        self.struct = s


class HeadIO:
    """A tenant's targets and outputs (device fp32 tensors)."""

    def __init__(self, targets, actions, loss, dW: list, db: list):
        self.targets, self.actions, self.loss, self.dW, self.db = targets, actions, loss, dW, db
        s = jn_head_io()
        s.targets = _ptr(targets)
        s.actions = _ptr(actions)
        s.loss = _ptr(loss)
        self._dW = (C.c_void_p * len(dW))(*[_ptr(w) for w in dW])
        self._db = (C.c_void_p * len(db))(*[_ptr(x) for x in db])
        s.dW = C.cast(self._dW, C.POINTER(C.c_void_p))
        s.db = C.cast(self._db, C.POINTER(C.c_void_p))
        self.struct = s


def _head_arrays(heads: Sequence[Head], ios: Sequence[HeadIO] = None):
    ha = (jn_head * len(heads))(*[h.struct for h in heads])
    ia = (jn_head_io * len(ios))(*[x.struct for x in ios]) if ios is not None else None
    return ha, ia


def jn_heads_workspace_size(packed: Packed, heads: Sequence[Head]) -> int:
    ha, _ = _head_arrays(heads)
    n = C.c_size_t()
    _check(_lib.jn_heads_workspace_size(C.byref(packed.struct), ha, len(heads), C.byref(n)),
           what="jn_heads_workspace_size")
    return int(n.value)


def jn_tenant_heads_fwd_bwd(ctx: Context, packed: Packed, hidden, heads: Sequence[Head], ios: Sequence[HeadIO],
                            ws, pooled=None):
    ha, ia = _head_arrays(heads, ios)
    _check(_lib.jn_tenant_heads_fwd_bwd(ctx.handle, C.byref(packed.struct), _ptr(hidden), ha, ia, len(heads),
                                        _ptr(ws), ws.numel() * ws.element_size(), _ptr(pooled)), ctx)


# Size of the library-owned workspace of the allocation-free heads call
# (JN_HEADS_SCRATCH_BYTES in joynexus.h).
HEADS_SCRATCH_BYTES = 64 << 20


def jn_tenant_heads_fwd_bwd_noalloc(ctx: Context, packed: Packed, hidden, heads: Sequence[Head],
                                    ios: Sequence[HeadIO], pooled=None):
    """The heads call on the library's own per-GPU scratch array (no
    workspace argument; allocates nothing)."""
    ha, ia = _head_arrays(heads, ios)
    _check(_lib.jn_tenant_heads_fwd_bwd_noalloc(ctx.handle, C.byref(packed.struct), _ptr(hidden), ha, ia,
                                                len(heads), _ptr(pooled)), ctx)


# ------------------------------------------------------- action expert ------

def jn_pack_tenant_sizes(reqs: Sequence[Request], tenants: Sequence[Tenant], d: int, align: int = 1):
    """(samples [G] int32, prefix rows [G] int64) of every tenant in the group."""
    ra, keep = _requests(reqs)
    ta = _tenants(tenants)
    G = len(tenants)
    n = np.zeros(G, np.int32)
    r = np.zeros(G, np.int64)
    _check(_lib.jn_pack_tenant_sizes(ra, len(reqs), ta, G, C.byref(_opts(d, align)),
                                     n.ctypes.data_as(C.POINTER(C.c_int32)),
                                     r.ctypes.data_as(C.POINTER(C.c_int64))), what="jn_pack_tenant_sizes")
    return n, r


class Expert:
    """A tenant's action expert: device bf16 tensors w_in [d, a], w_out [a, d],
    gf [d] and per layer a dict with the keys of ``EXPERT_LAYER_FIELDS``."""

    def __init__(self, w_in, w_out, gf, layers: List[dict], n_heads: int, chunk: int, d_prefix: int, eps: float,
                 w_time=None):
        self.w_in, self.w_out, self.gf, self.layers, self.w_time = w_in, w_out, gf, layers, w_time
        s = jn_expert()
        s.n_layers = len(layers)
        s.d = int(w_in.shape[0])
        s.n_heads = int(n_heads)
        s.ffn = int(layers[0]["w_up"].shape[0])
        s.action_dim = int(w_in.shape[1])
        s.chunk = int(chunk)
        s.d_prefix = int(d_prefix)
        s.eps = float(eps)
        s.w_in, s.w_out, s.gf = _ptr(w_in), _ptr(w_out), _ptr(gf)
        if w_time is not None:  # flow matching: [d, d_time] flow-time projection
            s.w_time = _ptr(w_time)
            s.d_time = int(w_time.shape[1])
        self._layers = (jn_expert_layer * len(layers))(
            *[jn_expert_layer(*[_ptr(lw[k]) for k in EXPERT_LAYER_FIELDS]) for lw in layers])
        s.layers = C.cast(self._layers, C.POINTER(jn_expert_layer))
        self.struct = s


class ExpertIO:
    """A tenant's expert inputs and outputs (device fp32 tensors): noisy /
    targets / pred [n, chunk, a], loss [1], dw_in, dw_out, dgf and per layer
    a dict of gradients keyed as ``EXPERT_LAYER_FIELDS``."""

    def __init__(self, n_samples: int, prefix_rows: int, noisy, targets, pred, loss, dw_in, dw_out, dgf,
                 layers: List[dict], flow_t=None, dw_time=None):
        self.noisy, self.targets, self.pred, self.loss = noisy, targets, pred, loss
        self.dw_in, self.dw_out, self.dgf, self.layers = dw_in, dw_out, dgf, layers
        self.flow_t, self.dw_time = flow_t, dw_time
        s = jn_expert_io()
        s.n_samples = int(n_samples)
        s.prefix_rows = int(prefix_rows)
        s.noisy, s.targets, s.pred, s.loss = _ptr(noisy), _ptr(targets), _ptr(pred), _ptr(loss)
        s.dw_in, s.dw_out, s.dgf = _ptr(dw_in), _ptr(dw_out), _ptr(dgf)
        s.flow_t, s.dw_time = _ptr(flow_t), _ptr(dw_time)
        self._layers = (jn_expert_layer_grads * len(layers))(
            *[jn_expert_layer_grads(*[_ptr(lg[k]) for k in EXPERT_LAYER_FIELDS]) for lg in layers])
        s.layers = C.cast(self._layers, C.POINTER(jn_expert_layer_grads))
        self.struct = s


def _expert_arrays(ex: Sequence[Expert], ios: Sequence[ExpertIO]):
    ea = (jn_expert * len(ex))(*[e.struct for e in ex])
    ia = (jn_expert_io * len(ios))(*[x.struct for x in ios])
    return ea, ia


def jn_experts_workspace_size(packed: Packed, ex: Sequence[Expert], ios: Sequence[ExpertIO]) -> int:
    ea, ia = _expert_arrays(ex, ios)
    n = C.c_size_t()
    _check(_lib.jn_experts_workspace_size(C.byref(packed.struct), ea, ia, len(ex), C.byref(n)),
           what="jn_experts_workspace_size")
    return int(n.value)


def jn_tenant_experts_fwd_bwd(ctx: Context, packed: Packed, hidden, ex: Sequence[Expert], ios: Sequence[ExpertIO],
                              ws):
    ea, ia = _expert_arrays(ex, ios)
    _check(_lib.jn_tenant_experts_fwd_bwd(ctx.handle, C.byref(packed.struct), _ptr(hidden), ea, ia, len(ex),
                                          _ptr(ws), ws.numel() * ws.element_size()), ctx)


# --------------------------------------------------------- token heads ------

class TokenHead:
    """A tenant's token head: device bf16 W [vocab, d]."""

    def __init__(self, W):
        if W.dtype is not _dtypes().bfloat16 or W.dim() != 2 or not W.is_contiguous():
            raise TypeError("W must be a contiguous bfloat16 tensor [vocab, d]")
        self.W, self.shape = W, tuple(W.shape)
        s = jn_token_head()
        s.vocab, s.W = int(W.shape[0]), W.data_ptr()
        self.struct = s


class TokenIO:
    """A tenant's targets (device int32 ``rows`` and ``targets`` [n]) and outputs: fp32 logp [n] and loss [1], bf16 or
    fp32 dW [vocab, d] and, optionally, bf16 dh [n, d]."""

    STRUCT = jn_token_io

    def __init__(self, rows, targets, logp, loss, dW, dh=None):
        t = _dtypes()
        self.rows, self.targets, self.logp, self.loss, self.dW, self.dh = rows, targets, logp, loss, dW, dh
        self.shape = tuple(dW.shape)  # of its head
        s = jn_token_io()
        n = s.n = int(rows.numel())
        s.rows = _entries("rows", rows, t.int32, n)
        s.targets = _entries("targets", targets, t.int32, n)
        s.logp = _entries("logp", logp, t.float32, n)
        s.loss = _entries("loss", loss, t.float32, 1)
        s.dw_f32 = 1 if dW.dtype is t.float32 else 0
        s.dW = _entries("dW", dW, t.float32 if s.dw_f32 else t.bfloat16, dW.numel())
        s.dh = _entries("dh", dh, t.bfloat16, n * int(dW.shape[1])) if dh is not None else None
        self.struct = s


class TokenPick:
    """Rows to decode (device int32 [n]) and outputs: token int32 [n], logp fp32 [n]."""

    STRUCT = jn_token_pick
    shape = None

    def __init__(self, rows, token, logp):
        t = _dtypes()
        self.rows, self.token, self.logp = rows, token, logp
        s = jn_token_pick()
        n = s.n = int(rows.numel())
        s.rows = _entries("rows", rows, t.int32, n)
        s.token = _entries("token", token, t.int32, n)
        s.logp = _entries("logp", logp, t.float32, n)
        self.struct = s


def _token_arrays(heads: Sequence[TokenHead], ios: Sequence, kind):
    G = len(heads)
    if G != len(ios) or G == 0:
        raise ValueError("one entry per token head")
    d = heads[0].shape[1]
    for h, io in zip(heads, ios):
        if h.shape[1] != d or (io.shape is not None and io.shape != h.shape) or type(io) is not kind:
            raise TypeError("token heads of one call share d, and dW has its W's shape")
    return d, G, (jn_token_head * G)(*[h.struct for h in heads]), (kind.STRUCT * G)(*[x.struct for x in ios])


def _tokens_size(call, heads, ios, kind) -> int:
    d, G, ha, ia = _token_arrays(heads, ios, kind)
    n = C.c_size_t()
    _check(call(d, ha, ia, G, C.byref(n)), what=call.__name__)
    return int(n.value)


def _tokens_call(call, ctx: Context, hidden, heads, ios, kind, ws):
    d, G, ha, ia = _token_arrays(heads, ios, kind)
    shape = hidden.shape
    if hidden.dtype is not _dtypes().bfloat16 or len(shape) != 2 or shape[1] != d or not hidden.is_contiguous():
        raise TypeError(f"hidden must be a contiguous bfloat16 tensor [T, {d}]")
    _check(call(ctx.handle, hidden.data_ptr(), shape[0], d, ha, ia, G, _ptr(ws), _bytes(ws)), ctx)


def jn_tokens_workspace_size(heads: Sequence[TokenHead], ios: Sequence[TokenIO]) -> int:
    return _tokens_size(_lib.jn_tokens_workspace_size, heads, ios, TokenIO)


def jn_tenant_tokens_fwd_bwd(ctx: Context, hidden, heads: Sequence[TokenHead], ios: Sequence[TokenIO], ws):
    _tokens_call(_lib.jn_tenant_tokens_fwd_bwd, ctx, hidden, heads, ios, TokenIO, ws)


def jn_tokens_decode_workspace_size(heads: Sequence[TokenHead], picks: Sequence[TokenPick]) -> int:
    return _tokens_size(_lib.jn_tokens_decode_workspace_size, heads, picks, TokenPick)


def jn_tenant_tokens_decode(ctx: Context, hidden, heads: Sequence[TokenHead], picks: Sequence[TokenPick], ws):
    _tokens_call(_lib.jn_tenant_tokens_decode, ctx, hidden, heads, picks, TokenPick, ws)


class TokenVerify:
    """A tenant's trees of drafted tokens (device int32 ``cu_nodes`` [trees + 1], ``tokens`` and ``parents`` [n], no
    parents: chains) and what they are held against: fp32 ``p`` [n, vocab] with the numbers ``u`` [n] and ``r`` [trees]
    and, where the drafts were drawn, their ``q`` [n, vocab]; or the likeliest tokens ``greedy`` [n].  Outputs, int32:
    ``path`` [trees, most nodes], ``n_path`` and ``next`` [trees]."""

    def __init__(self, cu_nodes, tokens, path, n_path, next, p=None, greedy=None, q=None, u=None, r=None, parents=None,
                 vocab: int = None):
        t = _dtypes()
        self.buffers = (cu_nodes, tokens, path, n_path, next, p, greedy, q, u, r, parents)
        s = jn_token_verify()
        n, trees = s.n, s.n_trees = int(tokens.numel()), int(cu_nodes.numel()) - 1
        if trees < 0 or path.dim() != 2:
            raise TypeError("cu_nodes must be [trees + 1], path [trees, most nodes]")
        s.max_path = int(path.shape[1])
        rows = lambda name, x: self._rows(name, x, n, t)  # noqa: E731
        if p is not None:
            s.p, s.ld_p = rows("p", p)
            s.u, s.r = _entries("u", u, t.float32, n), _entries("r", r, t.float32, trees)
        if q is not None:
            s.q, s.ld_q = rows("q", q)
        if (p is None and vocab is None) or (p is not None and q is not None and p.shape != q.shape):
            raise TypeError("p and q must be of one vocabulary; without p it is to be named")
        s.vocab = int(vocab if vocab is not None else p.shape[1])
        if p is not None and s.vocab > p.shape[1]:
            raise TypeError(f"p holds {p.shape[1]} probabilities, not {s.vocab}")
        s.cu_nodes = _entries("cu_nodes", cu_nodes, t.int32, trees + 1)
        s.tokens = _entries("tokens", tokens, t.int32, n)
        s.greedy = _entries("greedy", greedy, t.int32, n) if greedy is not None else None
        s.parents = _entries("parents", parents, t.int32, n) if parents is not None else None
        s.path = _entries("path", path, t.int32, trees * s.max_path)
        s.n_path, s.next = _entries("n_path", n_path, t.int32, trees), _entries("next", next, t.int32, trees)
        self.struct = s

    @staticmethod
    def _rows(name, x, n, t):
        if x.dtype is not t.float32 or x.dim() != 2 or x.shape[0] != n or (x.stride(1) != 1 and x.shape[1] > 1):
            raise TypeError(f"{name} must be a float32 tensor [{n}, vocab] of adjacent columns")
        if n > 1 and x.stride(0) < x.shape[1]:
            raise TypeError(f"rows of {name} overlap")
        return x.data_ptr(), x.stride(0) if n > 1 else x.shape[1]


def _verify_array(ios: Sequence[TokenVerify]):
    return (jn_token_verify * len(ios))(*[x.struct for x in ios]), len(ios)


def jn_tokens_verify_workspace_size(ios: Sequence[TokenVerify]) -> int:
    n = C.c_size_t()
    _check(_lib.jn_tokens_verify_workspace_size(*_verify_array(ios), C.byref(n)), what="jn_tokens_verify_workspace_size")
    return int(n.value)


def jn_tenant_tokens_verify(ctx: Context, ios: Sequence[TokenVerify], ws):
    _check(_lib.jn_tenant_tokens_verify(ctx.handle, *_verify_array(ios), _ptr(ws), _bytes(ws)), ctx)


# ---------------------------------------------------- tenant optimizer ------

class AdamWTenant:
    """One tenant's AdamW step: lists of device fp32 tensors (params, grads,
    first and second moments), optional bf16 copies (None entries allowed),
    hyperparameters and the 1-based index of this step."""

    def __init__(self, params: list, grads: list, m: list, v: list, step: int, lr: float, beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0, bf16_out: Optional[list] = None):
        self.tensors = (params, grads, m, v, bf16_out)
        n = len(params)
        import torch
        if not (len(grads) == len(m) == len(v) == n) or (bf16_out is not None and len(bf16_out) != n):
            raise ValueError("params, grads, m, v (and bf16_out) must have one entry per tensor")
        for i in range(n):
            for name, t in (("params", params[i]), ("grads", grads[i]), ("m", m[i]), ("v", v[i])):
                if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() != params[i].numel():
                    raise TypeError(f"{name}[{i}] must be a contiguous float32 tensor of {params[i].numel()} elements")
            if bf16_out is not None and bf16_out[i] is not None:
                b = bf16_out[i]
                if b.dtype != torch.bfloat16 or not b.is_contiguous() or b.numel() != params[i].numel():
                    raise TypeError(f"bf16_out[{i}] must be a contiguous bfloat16 tensor of {params[i].numel()} elements")
        s = jn_adamw_tenant()
        s.lr, s.beta1, s.beta2, s.eps, s.weight_decay = float(lr), float(beta1), float(beta2), float(eps), float(weight_decay)
        s.n_tensors = n
        s.step = int(step)
        mk = lambda xs: (C.c_void_p * max(n, 1))(*[_ptr(x) for x in xs])  # noqa: E731
        self._p, self._g, self._m, self._v = mk(params), mk(grads), mk(m), mk(v)
        self._n = (C.c_int64 * max(n, 1))(*[int(x.numel()) for x in params])
        s.params = C.cast(self._p, C.POINTER(C.c_void_p))
        s.grads = C.cast(self._g, C.POINTER(C.c_void_p))
        s.m = C.cast(self._m, C.POINTER(C.c_void_p))
        s.v = C.cast(self._v, C.POINTER(C.c_void_p))
        s.numel = C.cast(self._n, C.POINTER(C.c_int64))
        if bf16_out is not None:
            self._b = (C.c_void_p * max(n, 1))(*[_ptr(x) if x is not None else None for x in bf16_out])
            s.bf16_out = C.cast(self._b, C.POINTER(C.c_void_p))
        self.struct = s


def jn_adamw_workspace_size(tenants: Sequence[AdamWTenant]) -> int:
    arr = (jn_adamw_tenant * len(tenants))(*[t.struct for t in tenants])
    n = C.c_size_t()
    _check(_lib.jn_adamw_workspace_size(arr, len(tenants), C.byref(n)), what="jn_adamw_workspace_size")
    return int(n.value)


def jn_tenant_adamw_step(ctx: Context, tenants: Sequence[AdamWTenant], ws):
    arr = (jn_adamw_tenant * len(tenants))(*[t.struct for t in tenants])
    _check(_lib.jn_tenant_adamw_step(ctx.handle, arr, len(tenants), _ptr(ws), ws.numel() * ws.element_size()), ctx)


# -------------------------------------------------------------- unpack ------

def jn_unpack(ctx: Context, packed: Packed, reqs: Sequence[Request], rows, row_bytes: int, outs: Sequence):
    ra, keep = _requests(reqs)
    oa = (C.c_void_p * len(outs))(*[_ptr(o) for o in outs])
    _check(_lib.jn_unpack(ctx.handle, C.byref(packed.struct), ra, len(reqs), _ptr(rows), int(row_bytes), oa), ctx)


# ------------------------------------------------ inference-side batching ---

class Collector:
    """The inference queue's FIFO-compatible-prefix collector (host only):
    ``jn_collector_create / submit / poll / status``."""

    def __init__(self, max_batch_samples: int, timeout_us: int):
        h = C.c_void_p()
        _check(_lib.jn_collector_create(C.byref(h), int(max_batch_samples), int(timeout_us)),
               what="jn_collector_create")
        self.handle = h

    def submit(self, request_id: int, prefix_sig: int, d_model: int, n_samples: int, arrival_us: int):
        _check(_lib.jn_collector_submit(self.handle, int(request_id), int(prefix_sig), int(d_model), int(n_samples),
                                        int(arrival_us)), what="jn_collector_submit")

    def poll(self, now_us: int, cap: int = 4096) -> list:
        """Request ids of the batch ready at ``now_us`` (empty if none)."""
        ids = (C.c_int64 * max(cap, 1))()
        n = C.c_int32()
        _check(_lib.jn_collector_poll(self.handle, int(now_us), ids, int(cap), C.byref(n)), what="jn_collector_poll")
        return list(ids[: n.value])

    def status(self):
        """(queued requests, time the current prefix becomes ready or -1)."""
        n, t = C.c_int32(), C.c_int64()
        _check(_lib.jn_collector_status(self.handle, C.byref(n), C.byref(t)), what="jn_collector_status")
        return int(n.value), int(t.value)

    def close(self):
        if self.handle:
            _lib.jn_collector_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def jn_infer_workspace_size(reqs: Sequence[Request], tenants: Sequence[Tenant], d: int, align: int, bb: Backbone,
                            heads: Sequence[Head], pos=None) -> int:
    ra, keep = _requests(reqs)
    ha, _ = _head_arrays(heads)
    o = _opts(d, align)
    n = C.c_size_t()
    s = bb.struct if pos is None else _backbone_of(bb, jn_pack_plan(reqs, tenants, d, align).T, pos)
    _check(_lib.jn_infer_workspace_size(ra, len(reqs), _tenants(tenants), len(tenants), C.byref(o),
                                        C.byref(s), ha, C.byref(n)), what="jn_infer_workspace_size")
    return int(n.value)


class InferPlan:
    """``jn_infer_plan_*``: a resident decode-only step over one physical batch
    (device buffers stay referenced here for the plan's lifetime; ``pos`` as in
    ``jn_backbone_forward``, read at every launch)."""

    def __init__(self, ctx: Context, reqs: Sequence[Request], tenants: Sequence[Tenant], d: int, align: int,
                 bb: Backbone, heads: Sequence[Head], actions: Sequence, ws, pos=None):
        s = bb.struct
        if pos is not None or getattr(bb, "pos", None) is not None:
            s = _backbone_of(bb, jn_pack_plan(reqs, tenants, d, align).T, pos)
            pos = bb.pos if pos is None else pos
        ra, keep = _requests(reqs)
        ha, _ = _head_arrays(heads)
        o = _opts(d, align)
        acts = (C.c_void_p * len(actions))(*[_ptr(a) for a in actions])
        h = C.c_void_p()
        _check(_lib.jn_infer_plan_create(ctx.handle, ra, len(reqs), _tenants(tenants), len(tenants), C.byref(o),
                                         C.byref(s), ha, acts, _ptr(ws), ws.numel() * ws.element_size(),
                                         C.byref(h)), ctx)
        self.handle = h
        self.ctx = ctx
        self._keep = (reqs, bb, pos, heads, actions, ws)

    def packed(self):
        """(jn_packed struct, hidden device pointer) of the plan's batch."""
        s = jn_packed()
        hid = C.c_void_p()
        _check(_lib.jn_infer_plan_packed(self.handle, C.byref(s), C.byref(hid)), what="jn_infer_plan_packed")
        return s, hid.value

    def launch(self):
        _check(_lib.jn_infer_plan_launch(self.ctx.handle, self.handle), self.ctx)

    def capture(self):
        _check(_lib.jn_infer_plan_capture(self.ctx.handle, self.handle), self.ctx)

    def replay(self):
        _check(_lib.jn_infer_plan_replay(self.ctx.handle, self.handle), self.ctx)

    def close(self):
        if self.handle:
            _lib.jn_infer_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
