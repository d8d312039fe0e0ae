"""ctypes binding of include/tns_layer.h (attention over event lists, what stands between two layers, distillation): same names, marshalling only.

The functions without the prefix take torch tensors, as those of train_binding.py do: they check them, allocate what they return on the tensors'
device and enqueue on its current stream.  They record nothing for autograd, and so refuse tensors that require gradients while it records, and those with tangents (a
torch.autograd.Function of the caller's may call them).
"""
from __future__ import annotations

import ctypes as C
import functools

from .binding import TnsError, _check, lib as _lib  # noqa: F401
from .train_binding import TNS_BF16, TNS_F32, TNS_NEWEST_FIRST, TNS_ZERO_BEYOND, _dtype_of, _ld, _on, _unrecorded, _want  # noqa: F401

TNS_CENTER = 1
EXPORTS = ["tns_attend_workspace", "tns_attend_run", "tns_attend_grad", "tns_block_run", "tns_block_workspace", "tns_block_grad", "tns_distill_workspace", "tns_distill"]

_vp, _i64, _i32, _f64 = C.c_void_p, C.c_int64, C.c_int32, C.c_double
_at = C.c_size_t           # a device address or a stream


class tns_attend(C.Structure):
    _fields_ = [("S", _i64), ("rows", _i64), ("num", _i64), ("heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32), ("buckets", _i32), ("flags", _i32),
                ("d_rowptr", _vp), ("d_q", _vp), ("d_k", _vp), ("d_v", _vp), ("ld_q", _i64), ("ld_k", _i64), ("ld_v", _i64), ("d_index", _vp), ("d_mask", _vp), ("d_t", _vp),
                ("d_ts", _vp), ("d_edges", _vp), ("d_table", _vp), ("scale", _f64)]


class tns_block(C.Structure):
    _fields_ = [("rows", _i64), ("dim", _i32), ("dtype", _i32), ("flags", _i32), ("reserved", _i32), ("d_x", _vp), ("d_branch", _vp), ("d_gate", _vp), ("ld_x", _i64),
                ("ld_branch", _i64), ("ld_gate", _i64), ("d_scale", _vp), ("d_post", _vp), ("d_pre", _vp), ("eps", _f64)]


class tns_distill_desc(C.Structure):
    _fields_ = [("B", _i64), ("V", _i64), ("K", _i32), ("dtype", _i32), ("d_logits", _vp), ("ld_logits", _i64), ("d_ids", _vp), ("d_teacher", _vp), ("d_lse", _vp),
                ("d_weight", _vp), ("temperature", _f64), ("scale", _f64)]


_ready = None


def lib():
    global _ready
    if _ready is None:
        L = _lib()
        size_p = C.POINTER(C.c_size_t)
        L.tns_attend_workspace.argtypes = [C.POINTER(tns_attend), size_p, size_p, size_p]
        L.tns_attend_run.argtypes = [C.POINTER(tns_attend), _at, _at, _at, C.c_size_t, _at]
        L.tns_attend_grad.argtypes = [C.POINTER(tns_attend), _at, _at, _at, _at, _at, _at, _at, C.c_size_t, _at]
        L.tns_block_run.argtypes = [C.POINTER(tns_block), _at, _at, _at]
        L.tns_block_workspace.argtypes = [_i64, _i32, size_p]
        L.tns_block_grad.argtypes = [C.POINTER(tns_block), _at, _i64, _at, _i64, _at, _at, _at, _at, _at, _at, _at, C.c_size_t, _at]
        L.tns_distill_workspace.argtypes = [_i64, _i64, _i32, size_p]
        L.tns_distill.argtypes = [C.POINTER(tns_distill_desc), _at, _at, _at, _at, C.c_size_t, _at]
        for n in EXPORTS:
            getattr(L, n).restype = C.c_int
        _ready = L
    return _ready


# ---- the C functions -----------------------------------------------------------------------------

def tns_attend_workspace(a: tns_attend):
    """(bytes of workspace of tns_attend_run, of tns_attend_grad, bytes of saved values)"""
    n = [C.c_size_t() for _ in range(3)]
    _check(lib().tns_attend_workspace(C.byref(a), *[C.byref(x) for x in n]), "tns_attend_workspace")
    return tuple(int(x.value) for x in n)


def tns_attend_run(a: tns_attend, d_out, d_saved, d_workspace, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(lib().tns_attend_run(C.byref(a), d_out or 0, d_saved or 0, d_workspace or 0, workspace_bytes, hip_stream or 0), "tns_attend_run")


def tns_attend_grad(a: tns_attend, d_saved, d_dout, d_dq, d_dk, d_dv, d_dtable, d_workspace, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(lib().tns_attend_grad(C.byref(a), d_saved or 0, d_dout or 0, d_dq or 0, d_dk or 0, d_dv or 0, d_dtable or 0, d_workspace or 0, workspace_bytes, hip_stream or 0),
           "tns_attend_grad")


def tns_block_run(b: tns_block, d_out, d_next, hip_stream: int = 0) -> None:
    _check(lib().tns_block_run(C.byref(b), d_out or 0, d_next or 0, hip_stream or 0), "tns_block_run")


def tns_block_workspace(rows: int, dim: int) -> int:
    n = C.c_size_t()
    _check(lib().tns_block_workspace(rows, dim, C.byref(n)), "tns_block_workspace")
    return int(n.value)


def tns_block_grad(b: tns_block, d_dout, ld_dout: int, d_dnext, ld_dnext: int, d_dx, d_dbranch, d_dgate, d_dscale, d_dpost, d_dpre, d_workspace, workspace_bytes: int,
                   hip_stream: int = 0) -> None:
    _check(lib().tns_block_grad(C.byref(b), d_dout or 0, ld_dout, d_dnext or 0, ld_dnext, d_dx or 0, d_dbranch or 0, d_dgate or 0, d_dscale or 0, d_dpost or 0, d_dpre or 0,
                                d_workspace or 0, workspace_bytes, hip_stream or 0), "tns_block_grad")


def tns_distill_workspace(B: int, V: int, K: int) -> int:
    n = C.c_size_t()
    _check(lib().tns_distill_workspace(B, V, K, C.byref(n)), "tns_distill_workspace")
    return int(n.value)


def tns_distill(d: tns_distill_desc, d_loss, d_rows, d_dlogits, d_workspace, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(lib().tns_distill(C.byref(d), d_loss or 0, d_rows or 0, d_dlogits or 0, d_workspace or 0, workspace_bytes, hip_stream or 0), "tns_distill")


# ---- the same on torch tensors ---------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _attend_bytes(S, rows, num, heads, kv_heads, head_dim, dtype, buckets):
    return tns_attend_workspace(tns_attend(S, rows, num, heads, kv_heads, head_dim, dtype, buckets))


_block_bytes = functools.lru_cache(maxsize=1024)(tns_block_workspace)
_distill_bytes = functools.lru_cache(maxsize=1024)(tns_distill_workspace)


def _like(t):
    """A tensor of t's shape and type, dense."""
    import torch
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)      # (the first takes half as long)


def _heads(name, t, shape, like):
    """The address and the row stride of a tensor [rows, heads, dim] whose rows may lie apart."""
    if t.dtype is not like.dtype or t.shape != shape or t.device != like.device:
        raise ValueError(f"{name}: {like.dtype} of shape {shape} on {like.device} is wanted, not {t.dtype} of {tuple(t.shape)} on {t.device}")
    rows, heads, dim = shape
    if t.is_contiguous() or rows <= 1 and t[0].is_contiguous():
        return t.data_ptr(), heads * dim
    if not ((t.stride(2) == 1 or dim <= 1) and (t.stride(1) == dim or heads <= 1)):
        raise ValueError(f"{name}: the heads of a row and their channels have to lie side by side")
    return t.data_ptr(), t.stride(0)


def _described(rowptr, q, k, v, t, ts, edges, table, index, mask, scale, newest_first):
    import torch
    if rowptr.dim() != 1 or rowptr.shape[0] < 1 or q.dim() != 3 or k.dim() != 3:
        raise ValueError("rowptr has the shape [lists + 1], q [lists, heads, head_dim], k and v [rows, kv_heads, head_dim]")
    dev, f32 = q.device, torch.float32
    S, (_, heads, dim), (have, kv_heads, _) = rowptr.shape[0] - 1, q.shape, k.shape
    rows = index.shape[0] if index is not None else have
    buckets = 0 if table is None else table.shape[0]
    if mask is not None and mask.dtype is torch.bool:
        mask = mask.view(torch.uint8)
    if table is None and edges is not None:
        raise ValueError("edges without a table")
    if (edges is None) != (buckets <= 1) and not (buckets == 1 and edges.numel() == 0):
        raise ValueError("edges: one fewer than the rows of the table")
    p_q, ld_q = _heads("q", q, (S, heads, dim), q)
    p_k, ld_k = _heads("k", k, (have, kv_heads, dim), q)
    p_v, ld_v = _heads("v", v, (have, kv_heads, dim), q)
    return tns_attend(S, rows, have if index is not None else 0, heads, kv_heads, dim, _dtype_of(q), buckets, TNS_ZERO_BEYOND | (TNS_NEWEST_FIRST if newest_first else 0),
                      _want("rowptr", rowptr, (S + 1,), torch.int64, dev), p_q, p_k, p_v, ld_q, ld_k, ld_v, _want("index", index, (rows,), torch.int32, dev),
                      _want("mask", mask, (rows,), torch.uint8, dev), _want("t", t, (S,), f32, dev), _want("ts", ts, (rows,), f32, dev),
                      _want("edges", edges, (max(buckets - 1, 0),), f32, dev), _want("table", table, (buckets, heads), f32, dev), dim ** -0.5 if scale is None else scale)


def _sizes(a):
    return _attend_bytes(a.S, a.rows, a.num, a.heads, a.kv_heads, a.head_dim, a.dtype, a.buckets)


def attend_run(rowptr, q, k, v, t=None, ts=None, edges=None, table=None, index=None, mask=None, scale=None, newest_first=False, save=False) -> dict:
    """Attention of the targets over the lists of ``rowptr`` (tns_attend_run): ``out`` [lists, heads, head_dim] and, with ``save``, what
    attend_grad needs (``saved``).  ``table`` [buckets, heads] is the bias by age, ``edges`` its borders; ages are t - ts, or without
    times the number of newer events.  ``index`` (int32): the events' rows of k and v.  ``mask`` (bool or uint8): False leaves an event
    out.  ``scale`` is head_dim^-0.5 unless given.  k, v, ts, index and mask may have more rows than the lists hold."""
    import torch
    _unrecorded(q, k, v, t, ts, edges, table)
    on, stream = _on(q)
    a = _described(rowptr, q, k, v, t, ts, edges, table, index, mask, scale, newest_first)
    run, _, saved = _sizes(a)
    out = dict(out=_like(q), saved=q.new_empty(saved, dtype=torch.uint8) if save else None)
    ws = q.new_empty(run, dtype=torch.uint8)
    with on:
        rc = lib().tns_attend_run(C.byref(a), out["out"].data_ptr(), out["saved"].data_ptr() if save else 0, ws.data_ptr(), run, stream)
    if rc:
        _check(rc, "tns_attend_run")
    return out


def attend_grad(rowptr, q, k, v, saved, dout, t=None, ts=None, edges=None, table=None, mask=None, scale=None, newest_first=False) -> dict:
    """Gradients ``dq``, ``dk``, ``dv`` and ``dtable`` (None without a table), given those by the outputs; the other arguments as given to
    attend_run, ``saved`` from its result.  Rows of dk and dv that no list holds are zero."""
    import torch
    _unrecorded(q, k, v, t, ts, edges, table, dout)
    on, stream = _on(q)
    a = _described(rowptr, q, k, v, t, ts, edges, table, None, mask, scale, newest_first)
    _, grad, size = _sizes(a)
    if saved is None:
        raise ValueError("saved: attend_run(save=True) returns it")
    p_saved = _want("saved", saved, (size,), torch.uint8, q.device)
    p_dout = _want("dout", dout, q.shape, q.dtype, q.device)
    out = dict(dq=_like(q), dk=_like(k), dv=_like(v), dtable=None if table is None else _like(table))
    ws = q.new_empty(grad, dtype=torch.uint8)
    with on:
        tns_attend_grad(a, p_saved, p_dout, out["dq"].data_ptr(), out["dk"].data_ptr(), out["dv"].data_ptr(), 0 if table is None else out["dtable"].data_ptr(), ws.data_ptr(),
                        grad, stream)
    return out


def _between(x, branch, gate, scale, post, pre, eps, center):
    import torch
    if x.dim() != 2:
        raise ValueError("x has the shape [rows, dim]")
    (rows, dim), dev, f32, shape = x.shape, x.device, torch.float32, x.shape
    return tns_block(rows, dim, _dtype_of(x), TNS_CENTER if center else 0, 0, _want("x", x, shape, x.dtype, dev, False), _want("branch", branch, shape, x.dtype, dev, False),
                     _want("gate", gate, shape, x.dtype, dev, False), _ld(x, dim), _ld(branch, dim), _ld(gate, dim), _want("scale", scale, (dim,), f32, dev),
                     _want("post", post, (dim,), f32, dev), _want("pre", pre, (dim,), f32, dev), eps)


def block_run(x, branch, gate=None, scale=None, post=None, pre=None, eps=1e-6, center=False) -> dict:
    """What stands between two layers (tns_block_run): ``out`` = x + scale sigmoid(gate) post norm(branch) and ``next`` = pre norm(out)
    (None without ``pre``).  Without ``post`` the branch is not normed."""
    _unrecorded(x, branch, gate, scale, post, pre)
    on, stream = _on(x)
    b = _between(x, branch, gate, scale, post, pre, eps, center)
    out = dict(out=_like(x), next=None if pre is None else _like(x))
    with on:
        rc = lib().tns_block_run(C.byref(b), out["out"].data_ptr(), 0 if pre is None else out["next"].data_ptr(), stream)
    if rc:
        _check(rc, "tns_block_run")
    return out


def block_grad(x, branch, dout=None, dnext=None, gate=None, scale=None, post=None, pre=None, eps=1e-6, center=False) -> dict:
    """Gradients ``dx``, ``dbranch``, ``dgate``, ``dscale``, ``dpost`` and ``dpre`` (None for what is not there), given those by ``out`` and ``next``
    of block_run; its other arguments again."""
    import torch
    _unrecorded(x, branch, gate, scale, post, pre, dout, dnext)
    on, stream = _on(x)
    b = _between(x, branch, gate, scale, post, pre, eps, center)
    p_dout, p_dnext = (_want(name, v, x.shape, x.dtype, x.device, False) for name, v in (("dout", dout), ("dnext", dnext)))
    out = dict(dx=_like(x), dbranch=_like(branch), dgate=None if gate is None else _like(gate), dscale=None if scale is None else _like(scale),
               dpost=None if post is None else _like(post), dpre=None if pre is None else _like(pre))
    need = _block_bytes(b.rows, b.dim)
    ws = x.new_empty(need, dtype=torch.uint8)
    p = lambda t: 0 if t is None else t.data_ptr()      # noqa: E731
    with on:
        tns_block_grad(b, p_dout, _ld(dout, b.dim), p_dnext, _ld(dnext, b.dim), p(out["dx"]), p(out["dbranch"]), p(out["dgate"]), p(out["dscale"]), p(out["dpost"]), p(out["dpre"]),
                       ws.data_ptr(), need, stream)
    return out


def distill(logits, ids, teacher, lse=None, weight=None, temperature=1.0, scale=1.0, grad=True) -> dict:
    """Distillation from a teacher's highest scores (tns_distill): ``loss`` (a scalar tensor), ``rows`` [B], the weighted losses, and ``dlogits``
    (None without ``grad``).  ``ids`` (int32) and ``teacher`` [B, K]; ``lse`` [B], over all the teacher's candidates, has the others' mass counted."""
    import torch
    _unrecorded(logits, teacher, lse, weight)
    on, stream = _on(logits)
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits has the shape [rows, candidates], ids [rows, K]")
    (B, V), K, dev, f32 = logits.shape, ids.shape[1], logits.device, torch.float32
    d = tns_distill_desc(B, V, K, _dtype_of(logits), _want("logits", logits, (B, V), logits.dtype, dev, False), _ld(logits, V), _want("ids", ids, (B, K), torch.int32, dev),
                         _want("teacher", teacher, (B, K), f32, dev), _want("lse", lse, (B,), f32, dev), _want("weight", weight, (B,), f32, dev), temperature, scale)
    need = _distill_bytes(B, V, K)
    out = dict(loss=logits.new_empty((), dtype=f32), rows=logits.new_empty(B, dtype=f32), dlogits=_like(logits) if grad else None)
    ws = logits.new_empty(need, dtype=torch.uint8)
    with on:
        rc = lib().tns_distill(C.byref(d), out["loss"].data_ptr(), out["rows"].data_ptr(), out["dlogits"].data_ptr() if grad else 0, ws.data_ptr(), need, stream)
    if rc:
        _check(rc, "tns_distill")
    return out
