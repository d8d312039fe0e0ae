"""ctypes binding of include/tns_train.h (recurrence over event lists, paired log-ratio loss, AdamW): same names, marshalling only.

The functions without the prefix take torch tensors: they check them, allocate what they return on the tensors' device and
enqueue on its current stream.  Strides other than those of the last dimension are free where the C interface has them.
They record nothing for autograd, and so refuse tensors that require gradients while it records (a torch.autograd.Function of the
caller's may call them); what they change in place (a state table, weights) has its version raised, as by an operation of torch.
"""
from __future__ import annotations

import ctypes as C
import functools

from .binding import TnsError, _check, lib as _lib  # noqa: F401

TNS_F32, TNS_BF16 = 0, 1
TNS_NEWEST_FIRST, TNS_ZERO_BEYOND = 1, 4
ADAMW_BLOCK = 256          # weights that share a scale of a state in 8 bits
EXPORTS = ["tns_recur_workspace", "tns_recur_run", "tns_recur_grad", "tns_recur_step", "tns_pair_loss_workspace", "tns_pair_loss",
           "tns_adamw_create", "tns_adamw_step", "tns_adamw_destroy"]

_vp, _i64, _i32, _f64 = C.c_void_p, C.c_int64, C.c_int32, C.c_double
_at = C.c_size_t           # a device address or a stream: an integer (a c_void_p argument would take bytes, strings and arrays, as addresses of host memory)


class tns_recur(C.Structure):
    _fields_ = [("S", _i64), ("rows", _i64), ("dim", _i32), ("dtype", _i32), ("flags", _i32), ("reserved", _i32), ("d_rowptr", _vp), ("d_u", _vp),
                ("d_x", _vp), ("ld_u", _i64), ("ld_x", _i64), ("d_ts", _vp), ("d_decay", _vp), ("d_h0", _vp), ("d_t0", _vp)]


class tns_pairs(C.Structure):
    _fields_ = [("B", _i64), ("K", _i64), ("dim", _i32), ("dtype", _i32), ("d_anchor", _vp), ("d_pos", _vp), ("d_neg", _vp), ("ld_anchor", _i64),
                ("ld_pos", _i64), ("d_ref", _vp), ("d_weight", _vp), ("beta", _f64), ("smoothing", _f64), ("scale", _f64)]


class tns_adamw_tensor(C.Structure):
    _fields_ = [("n", _i64), ("d_param", _vp), ("d_copy", _vp), ("d_grad", _vp), ("d_m", _vp), ("d_v", _vp), ("d_m_scale", _vp), ("d_v_scale", _vp),
                ("weight_decay", _f64)]


class tns_adamw_config(C.Structure):
    _fields_ = [("beta1", _f64), ("beta2", _f64), ("eps", _f64), ("seed", C.c_uint64), ("state_bits", _i32), ("grad_dtype", _i32), ("device", _i32),
                ("reserved", _i32)]


_ready = False


def lib():
    global _ready
    L = _lib()
    if not _ready:
        size_p = C.POINTER(C.c_size_t)
        L.tns_recur_workspace.argtypes = [C.POINTER(tns_recur), size_p, size_p, size_p]
        L.tns_recur_run.argtypes = [C.POINTER(tns_recur), _at, _i64, _at, _at, _at, C.c_size_t, _at]
        L.tns_recur_grad.argtypes = [C.POINTER(tns_recur), _at, _at, _i64, _at, _at, _i64, _at, _i64, _at, _at, _at, C.c_size_t, _at]
        L.tns_recur_step.argtypes = [_i64, _i64, _i32, _i32, _at, _at, _i64, _at, _i64, _at, _at, _at, _at, _at, _i64, _at]
        L.tns_pair_loss_workspace.argtypes = [_i64, _i64, _i32, size_p]
        L.tns_pair_loss.argtypes = [C.POINTER(tns_pairs), _at, _at, _at, _at, _at, _at, C.c_size_t, _at]
        L.tns_adamw_create.argtypes = [C.POINTER(tns_adamw_config), _i32, C.POINTER(tns_adamw_tensor), C.POINTER(_vp)]
        L.tns_adamw_step.argtypes = [_vp, _f64, _i64, _at, _at]
        L.tns_adamw_destroy.argtypes = [_vp]
        for n in EXPORTS:
            getattr(L, n).restype = C.c_int
        _ready = True
    return L


# ---- the C functions -----------------------------------------------------------------------------

def tns_recur_workspace(r: tns_recur):
    """(bytes of workspace of tns_recur_run, of tns_recur_grad, bytes of saved states)"""
    n = [C.c_size_t() for _ in range(3)]
    _check(lib().tns_recur_workspace(C.byref(r), *[C.byref(x) for x in n]), "tns_recur_workspace")
    return tuple(int(x.value) for x in n)


def tns_recur_run(r: tns_recur, d_h, ld_h: int, d_h_last, d_saved, d_workspace, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(lib().tns_recur_run(C.byref(r), d_h or 0, ld_h, d_h_last or 0, d_saved or 0, d_workspace or 0, workspace_bytes, hip_stream or 0),
           "tns_recur_run")


def tns_recur_grad(r: tns_recur, d_saved, d_dh, ld_dh: int, d_dh_last, d_du, ld_du: int, d_dx, ld_dx: int, d_ddecay, d_dh0, d_workspace,
                   workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(lib().tns_recur_grad(C.byref(r), d_saved or 0, d_dh or 0, ld_dh, d_dh_last or 0, d_du or 0, ld_du, d_dx or 0, ld_dx,
                                d_ddecay or 0, d_dh0 or 0, d_workspace or 0, workspace_bytes, hip_stream or 0), "tns_recur_grad")


def tns_recur_step(B: int, num_ids: int, dim: int, dtype: int, d_ids, d_u, ld_u: int, d_x, ld_x: int, d_ts, d_decay, d_state, d_state_ts, d_out,
                   ld_out: int, hip_stream: int = 0) -> None:
    _check(lib().tns_recur_step(B, num_ids, dim, dtype, d_ids or 0, d_u or 0, ld_u, d_x or 0, ld_x, d_ts or 0, d_decay or 0,
                                d_state or 0, d_state_ts or 0, d_out or 0, ld_out, hip_stream or 0), "tns_recur_step")


def tns_pair_loss_workspace(B: int, K: int, dim: int) -> int:
    n = C.c_size_t()
    _check(lib().tns_pair_loss_workspace(B, K, dim, C.byref(n)), "tns_pair_loss_workspace")
    return int(n.value)


def tns_pair_loss(p: tns_pairs, d_loss, d_margin, d_danchor, d_dpos, d_dneg, d_workspace, workspace_bytes: int, hip_stream: int = 0) -> None:
    _check(lib().tns_pair_loss(C.byref(p), d_loss or 0, d_margin or 0, d_danchor or 0, d_dpos or 0, d_dneg or 0, d_workspace or 0,
                               workspace_bytes, hip_stream or 0), "tns_pair_loss")


def tns_adamw_create(cfg: tns_adamw_config, tensors):
    table = (tns_adamw_tensor * len(tensors))(*tensors)
    h = _vp()
    _check(lib().tns_adamw_create(C.byref(cfg), len(tensors), table, C.byref(h)), "tns_adamw_create")
    return h


def tns_adamw_step(opt, lr: float, t: int, d_grad_scale=None, hip_stream: int = 0) -> None:
    _check(lib().tns_adamw_step(opt, lr, t, d_grad_scale or 0, hip_stream or 0), "tns_adamw_step")


def tns_adamw_destroy(opt) -> None:
    _check(lib().tns_adamw_destroy(opt), "tns_adamw_destroy")


# ---- the same on torch tensors ---------------------------------------------------------------------

def _unrecorded(*tensors):
    """Refuses what autograd would have to follow: the results would look like constants to it."""
    for t in tensors:
        if t is not None and t.requires_grad:
            import torch
            if torch.is_grad_enabled():
                raise ValueError("nothing is recorded for autograd here: call under torch.no_grad(), within a torch.autograd.Function, or on detached tensors")


def _dtype_of(t):
    import torch
    if t.dtype is torch.float32:
        return TNS_F32
    if t.dtype is torch.bfloat16:
        return TNS_BF16
    raise ValueError(f"float32 or bfloat16 is wanted, not {t.dtype}")


def _want(name, t, shape, dtype, device, dense=True):
    """The address of a tensor of that shape and type, 0 for None; rows of a matrix may lie apart where it need not be dense."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.device != device:
        raise ValueError(f"{name}: {dtype} of shape {tuple(shape)} on {device} is wanted, not {t.dtype} of {tuple(t.shape)} on {t.device}")
    if not t.is_contiguous() and (dense or not (t.stride(-1) == 1 or t.shape[-1] <= 1)):
        raise ValueError(f"{name}: " + ("a contiguous tensor is wanted" if dense else "the channels of a row have to lie side by side"))
    return t.data_ptr()


def _ld(t, dim):
    return dim if t is None or t.shape[0] <= 1 else t.stride(0)


class _Here:
    """Leaves the current device as it is."""

    def __enter__(self):
        pass

    def __exit__(self, *_):
        pass


_HERE = _Here()


def _on(t):
    """A context in which a tensor's GPU is the current one, and its current stream."""
    import torch
    if not t.is_cuda:
        raise ValueError("tensors on the GPU are wanted")
    index = t.device.index
    return _HERE if torch.cuda.current_device() == index else torch.cuda.device(index), torch.cuda.current_stream(index).cuda_stream


@functools.lru_cache(maxsize=1024)
def _recur_bytes(S, rows, dim, dtype):
    return tns_recur_workspace(tns_recur(S, rows, dim, dtype))


_pair_bytes = functools.lru_cache(maxsize=1024)(tns_pair_loss_workspace)


def _lists(rowptr, u, x, ts, decay, h0, t0, newest_first):
    import torch
    if u.dim() != 2 or rowptr.dim() != 1 or rowptr.shape[0] < 1:
        raise ValueError("u has the shape [rows, dim], rowptr [lists + 1]")
    shape, S, dev, f32 = u.shape, rowptr.shape[0] - 1, u.device, torch.float32
    rows, dim = shape
    dtype = _dtype_of(u)
    return tns_recur(S, rows, dim, dtype, TNS_NEWEST_FIRST if newest_first else 0, 0, _want("rowptr", rowptr, (S + 1,), torch.int64, dev),
                     _want("u", u, shape, u.dtype, dev, False), _want("x", x, shape, u.dtype, dev, False), _ld(u, dim), _ld(x, dim),
                     _want("ts", ts, (rows,), f32, dev), _want("decay", decay, (dim,), f32, dev), _want("h0", h0, (S, dim), f32, dev),
                     _want("t0", t0, (S,), f32, dev))


def recur_run(rowptr, u, x, ts=None, decay=None, h0=None, t0=None, newest_first=False, states=True, save=False) -> dict:
    """The recurrence over the lists of ``rowptr`` (tns_recur_run): ``h`` (None without ``states``), ``last`` and, with ``save``,
    what recur_grad needs (``saved``).  u and x may have more rows than the lists hold: those of ``h`` are zero."""
    import torch
    _unrecorded(u, x, ts, decay, h0, t0)
    on, stream = _on(u)
    r = _lists(rowptr, u, x, ts, decay, h0, t0, newest_first)
    r.flags |= TNS_ZERO_BEYOND
    run, _, saved = _recur_bytes(r.S, r.rows, r.dim, r.dtype)
    out = dict(h=u.new_empty((r.rows, r.dim)) if states else None, last=u.new_empty((r.S, r.dim), dtype=torch.float32),
               saved=u.new_empty(saved, dtype=torch.uint8) if save else None)
    ws = u.new_empty(run, dtype=torch.uint8)
    with on:
        tns_recur_run(r, out["h"].data_ptr() if states else 0, r.dim, out["last"].data_ptr(), out["saved"].data_ptr() if save else 0, ws.data_ptr(), run, stream)
    return out


def recur_grad(rowptr, u, x, saved, ts=None, decay=None, h0=None, t0=None, newest_first=False, dh=None, dlast=None) -> dict:
    """Gradients ``du``, ``dx``, ``ddecay`` (None without decay) and ``dh0`` (None without h0), given those by the states (``dh``)
    and by the last states (``dlast``); the other arguments as given to recur_run, ``saved`` from its result.  Rows of du and dx that
    no list holds are zero."""
    import torch
    _unrecorded(u, x, ts, decay, h0, t0, dh, dlast)
    on, stream = _on(u)
    r = _lists(rowptr, u, x, ts, decay, h0, t0, newest_first)
    r.flags |= TNS_ZERO_BEYOND
    _, grad, size = _recur_bytes(r.S, r.rows, r.dim, r.dtype)
    if saved is None:
        raise ValueError("saved: recur_run(save=True) returns it")
    p_saved = _want("saved", saved, (size,), torch.uint8, u.device)
    p_dh = _want("dh", dh, u.shape, u.dtype, u.device, False)
    p_dlast = _want("dlast", dlast, (r.S, r.dim), torch.float32, u.device)
    out = dict(du=u.new_empty((r.rows, r.dim)), dx=u.new_empty((r.rows, r.dim)), ddecay=u.new_empty(r.dim, dtype=torch.float32) if decay is not None else None,
               dh0=u.new_empty((r.S, r.dim), dtype=torch.float32) if h0 is not None else None)
    ws = u.new_empty(grad, dtype=torch.uint8)
    p = lambda t: 0 if t is None else t.data_ptr()      # noqa: E731
    with on:
        tns_recur_grad(r, p_saved, p_dh, _ld(dh, r.dim), p_dlast, p(out["du"]), r.dim, p(out["dx"]), r.dim, p(out["ddecay"]), p(out["dh0"]), ws.data_ptr(),
                       grad, stream)
    return out


def recur_step(ids, u, x, state, ts=None, decay=None, state_ts=None):
    """One event for each node of ``ids`` (int32, distinct): changes ``state`` (and ``state_ts``) in place, returns the new states
    in u's type, zero for ids that hold none."""
    import torch
    _unrecorded(u, x, state, ts, decay, state_ts)
    on, stream = _on(u)
    if u.dim() != 2 or state.dim() != 2:
        raise ValueError("u has the shape [events, dim], state [nodes, dim]")
    shape, n, dev, f32 = u.shape, state.shape[0], u.device, torch.float32
    B, dim = shape
    dtype = _dtype_of(u)
    out = u.new_empty((B, dim))
    args = (_want("ids", ids, (B,), torch.int32, dev), _want("u", u, shape, u.dtype, dev, False), _ld(u, dim),
            _want("x", x, shape, u.dtype, dev, False), _ld(x, dim), _want("ts", ts, (B,), f32, dev), _want("decay", decay, (dim,), f32, dev),
            _want("state", state, (n, dim), f32, dev), _want("state_ts", state_ts, (n,), f32, dev))
    with on:
        tns_recur_step(B, n, dim, dtype, *args, out.data_ptr(), dim, stream)
    torch.autograd.graph.increment_version([state] if state_ts is None else [state, state_ts])
    return out


def pair_loss(anchor, pos, neg, ref=None, weight=None, beta=1.0, smoothing=0.0, scale=1.0, grads=True) -> dict:
    """Paired log-ratio loss (tns_pair_loss): ``loss`` (a scalar tensor), ``margin`` [B, K] and the gradients ``danchor``, ``dpos``,
    ``dneg`` (None without ``grads``)."""
    import torch
    _unrecorded(anchor, pos, neg, ref, weight)
    on, stream = _on(anchor)
    if neg.dim() != 3:
        raise ValueError("neg has the shape [events, links, dim]")
    (B, K, dim), dev, dt, f32 = neg.shape, anchor.device, anchor.dtype, torch.float32
    p = tns_pairs(B, K, dim, _dtype_of(anchor), _want("anchor", anchor, (B, dim), dt, dev, False), _want("pos", pos, (B, dim), dt, dev, False),
                  _want("neg", neg, neg.shape, dt, dev), _ld(anchor, dim), _ld(pos, dim), _want("ref", ref, (B, K), f32, dev),
                  _want("weight", weight, (B, K), f32, dev), beta, smoothing, scale)
    need = _pair_bytes(B, K, dim)
    loss, margin, ws = anchor.new_empty((), dtype=f32), anchor.new_empty((B, K), dtype=f32), anchor.new_empty(need, dtype=torch.uint8)
    da, dp, dn = (anchor.new_empty((B, dim)), anchor.new_empty((B, dim)), anchor.new_empty((B, K, dim))) if grads else (None,) * 3
    g = (da.data_ptr(), dp.data_ptr(), dn.data_ptr()) if grads else (0, 0, 0)
    with on:
        tns_pair_loss(p, loss.data_ptr(), margin.data_ptr(), *g, ws.data_ptr(), need, stream)
    return dict(loss=loss, margin=margin, danchor=da, dpos=dp, dneg=dn)


class AdamW:
    """Owns a tns_adamw over lists of contiguous tensors that stay where they are: ``params`` (float32), ``grads`` (all float32 or all
    bfloat16) and, where given, bfloat16 ``copies`` that receive the new weights.  ``weight_decay`` is one number or one for each
    tensor.  ``states``: (m, v) or, in 8 bits, (m, v, m_scale, v_scale), lists of tensors that continue an earlier run; zeros
    otherwise.  They are the attributes of the same names; the codes of 8-bit states are torch.float8_e4m3fn, v's of its root."""

    def __init__(self, params, grads, copies=None, bits=32, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, seed=0, states=None):
        import torch
        if not params or len(grads) != len(params) or (copies is not None and len(copies) != len(params)):
            raise ValueError("one gradient (and copy) for each tensor is wanted, and one tensor at least")
        if bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        dev, kind = params[0].device, torch.float8_e4m3fn if bits == 8 else torch.float32
        if dev.type != "cuda":
            raise ValueError("tensors on the GPU are wanted")
        blocks = [-(-p.numel() // ADAMW_BLOCK) for p in params]
        if states is None:
            states = [[torch.zeros(p.shape, dtype=kind, device=dev) for p in params] for _ in range(2)]
            states += [[torch.zeros(b, dtype=torch.float32, device=dev) for b in blocks] for _ in range(2)] if bits == 8 else [None, None]
        self.m, self.v, self.m_scale, self.v_scale = (list(states) + [None, None])[:4]
        self.params, self.grads, self.copies, self.bits = list(params), list(grads), copies, bits
        decays = [float(weight_decay)] * len(params) if not hasattr(weight_decay, "__len__") else [float(d) for d in weight_decay]
        if len(decays) != len(params):
            raise ValueError("one weight_decay for each tensor is wanted")
        table = []
        for i, p in enumerate(params):
            at = lambda name, many, dtype, shape: 0 if many is None else _want(f"{name}[{i}]", many[i], shape, dtype, dev)      # noqa: E731
            shape, scales = tuple(p.shape), (blocks[i],)
            table.append(tns_adamw_tensor(p.numel(), at("params", params, torch.float32, shape), at("copies", copies, torch.bfloat16, shape),
                                          at("grads", grads, grads[0].dtype, shape), at("m", self.m, kind, shape), at("v", self.v, kind, shape),
                                          at("m_scale", self.m_scale, torch.float32, scales), at("v_scale", self.v_scale, torch.float32, scales), decays[i]))
        cfg = tns_adamw_config(betas[0], betas[1], eps, seed & (1 << 64) - 1, bits, _dtype_of(grads[0]), dev.index, 0)
        self._device = dev
        changed = [t for many in (params, copies, self.m, self.v, self.m_scale, self.v_scale) if many is not None for t in many]
        self._changed = list({id(t if t._base is None else t._base): t for t in changed}.values())      # (views of one tensor have one version)
        self._h = tns_adamw_create(cfg, table)

    def step(self, lr, t, grad_scale=None):
        """Step number ``t`` (from 1 on); ``grad_scale``: a float32 tensor of one value that the gradients are multiplied with."""
        import torch
        scale = 0 if grad_scale is None else _want("grad_scale", grad_scale.reshape(-1), (1,), torch.float32, self._device)
        tns_adamw_step(self._h, lr, t, scale, torch.cuda.current_stream(self._device).cuda_stream)
        torch.autograd.graph.increment_version(self._changed)

    def close(self):
        if getattr(self, "_h", None):
            tns_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
