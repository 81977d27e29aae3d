"""Operators of a recurrent model's block (include/comba_block.h): linear attention
with a decay for each head, and the norms after and before a block fused with its
gate, residual scale and residual stream.

    o, ht = comba_decay_fwd(q, k, v, g, h0)             # prompts; comba_decay_step: one token
    r, n = comba_block_norm_fwd(y, x, weight, post_weight=w1, z=z, scale=s)

and, differentiable (torch.autograd), comba_decay and comba_block_norm.  Types, slices, packed sequences,
streams and workspaces are those of the layer's operators (``layer.py``).
"""
from __future__ import annotations

import ctypes
import struct

from . import COMBA_BF16, COMBA_F32, CombaError, _kept_offsets, _ptr, load_library
from .layer import (_NORM_ACT, _SCAN_ROW, _activation, _code, _dense, _host_ptr, _like, _memory, _on, _row, _run, _seqs,
                    _slots, _workspace)

__all__ = ["comba_decay_fwd", "comba_decay_fwd_save", "comba_decay_bwd", "comba_decay_step",
           "comba_decay", "comba_block_norm_fwd", "comba_block_norm_bwd", "comba_block_norm",
           "CombaDecayShape", "CombaBlockNormShape"]

_I32, _I64, _P = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class CombaDecayShape(ctypes.Structure):
    _fields_ = [("B", _I32), ("T", _I32), ("H", _I32), ("Hq", _I32), ("Hk", _I32), ("Hv", _I32),
                ("dk", _I32), ("dv", _I32), ("num_seqs", _I32), ("cu_seqlens", _P),
                ("cu_seqlens_host", _P), ("in_dtype", ctypes.c_int), ("g_dtype", ctypes.c_int),
                ("g_per_head", _I32), ("scale", ctypes.c_float), ("q_row", _I64),
                ("k_row", _I64), ("v_row", _I64), ("g_row", _I64)]


class CombaBlockNormShape(ctypes.Structure):
    _fields_ = [("rows", _I64), ("C", _I32), ("dtype", ctypes.c_int), ("x_dtype", ctypes.c_int),
                ("activation", ctypes.c_int), ("eps", ctypes.c_float), ("y_row", _I64),
                ("z_row", _I64), ("x_row", _I64)]


_DECAY = struct.Struct("@iiiiiiiiiPPiiifqqqq")
_NORM = struct.Struct("@qiiiifqqq")
assert _NORM.size == ctypes.sizeof(CombaBlockNormShape)
assert _DECAY.size == ctypes.sizeof(CombaDecayShape)


def bind(lib):
    """Declare the C signatures (called by load_library); the shape structs pass as bytes."""
    P, Z, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    for name, args in (("comba_decay_fwd", [P] * 9 + [Z, P]),
                       ("comba_decay_fwd_save", [P] * 9 + [Z, P]),
                       ("comba_decay_bwd", [P] * 14 + [Z, P, Z, P]),
                       ("comba_decay_step", [P] * 7 + [_I32, P, P]),
                       ("comba_block_norm_fwd", [P] * 10),
                       ("comba_block_norm_bwd", [P] * 16 + [Z, P])):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, I
    for name in ("comba_decay_fwd_workspace_bytes", "comba_decay_save_bytes",
                 "comba_decay_bwd_workspace_bytes", "comba_block_norm_workspace_bytes"):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = [P], Z


# ---- linear attention with a decay per head ------------------------------------------
def _heads(name, t, lead, first, dtype, dev, far):
    """(heads, head size, elements between token rows) of q, k or v."""
    shape = t.shape
    if len(shape) != lead + 2 or shape[:lead] != first or t.dtype is not dtype \
            or t.get_device() != dev:
        raise CombaError("comba: %s must be %s %s on the device"
                         % (name, str(dtype).replace("torch.", ""), list(first) + ["heads", "d"]))
    h, d = shape[-2], shape[-1]
    if t.is_contiguous():
        return h, d, 0
    if lead == 1:  # (a step's common slice, without the general check's loops)
        row, head, one = t.stride()
        if one == 1 and head == d and row >= h * d:
            return h, d, row
    return h, d, _row(name, t, lead, shape, dtype, dev, far)


def _decay_shape(lead, q, k, v, g, scale, N, cu, host):
    """(shape struct, pointers, (H, dk, dv)) of a call whose tensors have ``lead`` leading
    dimensions of tokens."""
    import torch

    code, dev, dt, f32 = _code(q, "q"), q.get_device(), q.dtype, torch.float32
    far = None if lead == 1 else _SCAN_ROW
    first, gs, gt = q.shape[:lead], g.shape, g.dtype
    Hq, dk, q_row = _heads("q", q, lead, first, dt, dev, far)
    Hk, dk2, k_row = _heads("k", k, lead, first, dt, dev, far)
    Hv, dv, v_row = _heads("v", v, lead, first, dt, dev, far)
    if dk != dk2:
        raise CombaError("comba: q and k must have one head size")
    per_head = len(gs) == 1
    if not per_head and (len(gs) != lead + 1 or gs[:lead] != first):
        raise CombaError("comba: g must be [..,H], or [H] for constants of the heads")
    H = gs[-1]
    if H < 1 or Hq < 1 or Hk < 1 or Hv < 1 or H % Hq or H % Hk or H % Hv:
        raise CombaError("comba: the heads of q, k and v must divide those of g")
    if not (1 <= dk <= 256 and 1 <= dv <= 256):
        raise CombaError("comba: head sizes must be 1..256")
    if gt is not f32 and (per_head or gt is not dt):
        raise CombaError("comba: g must be float32%s" % ("" if per_head else ", or of q's dtype"))
    if per_head:
        _dense("g", g, gs, f32, dev)
    shp = _DECAY.pack(first[0], 1 if lead == 1 else first[1], H, Hq, Hk, Hv, dk, dv, N, cu,
                      _host_ptr(host), code, COMBA_F32 if gt is f32 else COMBA_BF16,
                      1 if per_head else 0, dk ** -0.5 if scale is None else scale, q_row, k_row,
                      v_row, 0 if per_head else _row("g", g, lead, first + (H,), gt, dev, far))
    return shp, (q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr()), (H, dk, dv), dev


def _outputs(v, H):
    """An uninitialised contiguous o: as v, with H heads."""
    return _like(v) if v.shape[-2] == H else v.new_empty(v.shape[:-2] + (H, v.shape[-1]))


def _decay(save, q, k, v, g, h0, scale, cu_seqlens, cu_seqlens_host, output_final_state,
           workspace, stream):
    import torch

    lib = load_library()
    _code(q, "q")
    if q.dim() != 4:
        raise CombaError("comba: q must be [B,T,heads,dk]")
    S, cu, host = _seqs(q.shape[0], cu_seqlens, cu_seqlens_host, q.get_device())
    shp, ptrs, (H, dk, dv), dev = _decay_shape(2, q, k, v, g, scale, S, cu, host)
    state = (S, H, dk, dv)
    h0p = _dense("h0", h0, state, torch.float32, dev)
    o = _outputs(v, H)
    ht = q.new_empty(state, dtype=torch.float32) if output_final_state else None
    ws = _workspace(lib.comba_decay_save_bytes if save else lib.comba_decay_fwd_workspace_bytes,
                    shp, workspace, q.device)
    fn = lib.comba_decay_fwd_save if save else lib.comba_decay_fwd
    _run(fn(shp, *ptrs, h0p, o.data_ptr(), _ptr(ht), ws.data_ptr(), ws.numel(),
            _on(stream, dev, o, ht, ws)))
    return o, ht, ws


def comba_decay_fwd(q, k, v, g, h0=None, *, scale=None, cu_seqlens=None, cu_seqlens_host=None,
                    output_final_state=True, workspace=None, stream=None):
    """Linear attention with a decay for each head.  Returns (o [B,T,H,dv], ht [S,H,dk,dv]
    float32 or None).

    S_t = exp(g_t) S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t  (scale: dk^-0.5 by default).
    q [B,T,Hq,dk], k [B,T,Hk,dk], v [B,T,Hv,dv] of one dtype and each possibly a column
    slice; g [B,T,H] (float32 or q's dtype, possibly a slice) or [H] float32, constants of
    the heads; Hq, Hk and Hv divide H, and neighbouring heads share one.  dk, dv: 1..256.
    h0 [S,H,dk,dv] float32.  Rows of a slice lie at most 2^22 elements apart."""
    o, ht, _ = _decay(False, q, k, v, g, h0, scale, cu_seqlens, cu_seqlens_host,
                      output_final_state, workspace, stream)
    return o, ht


def comba_decay_fwd_save(q, k, v, g, h0=None, *, scale=None, cu_seqlens=None,
                         cu_seqlens_host=None, output_final_state=True, workspace=None,
                         stream=None):
    """comba_decay_fwd that also keeps the states its backward needs.  Returns (o, ht,
    workspace); pass the same inputs and ``workspace`` to comba_decay_bwd."""
    return _decay(True, q, k, v, g, h0, scale, cu_seqlens, cu_seqlens_host, output_final_state,
                  workspace, stream)


def comba_decay_bwd(q, k, v, g, h0, do, dht=None, *, workspace, scale=None, cu_seqlens=None,
                    cu_seqlens_host=None, need_dg=True, need_dh0=True, scratch=None, stream=None):
    """Backward of comba_decay_fwd_save from do [B,T,H,dv] (dtype of q) and dht [S,H,dk,dv]
    float32, with the ``workspace`` it filled (either call may know the offsets on the host);
    ``scratch``: memory for the call itself, made if absent.  Returns dict dq, dk, dv (dtype of
    q), dg (dtype of g; None for constants of the heads), dh0 (float32)."""
    import torch

    lib = load_library()
    _code(q, "q")
    if q.dim() != 4:
        raise CombaError("comba: q must be [B,T,heads,dk]")
    S, cu, host = _seqs(q.shape[0], cu_seqlens, cu_seqlens_host, q.get_device())
    shp, ptrs, (H, dk, dv), dev = _decay_shape(2, q, k, v, g, scale, S, cu, host)
    state = (S, H, dk, dv)
    given = (_dense("h0", h0, state, torch.float32, dev),
             _dense("do", do, q.shape[:2] + (H, dv), q.dtype, dev),
             _dense("dht", dht, state, torch.float32, dev))
    out = {"dq": _like(q), "dk": _like(k), "dv": _like(v),
           "dg": _like(g) if need_dg and g.dim() == 3 else None,
           "dh0": q.new_empty(state, dtype=torch.float32) if need_dh0 else None}
    if workspace is None:
        raise CombaError("comba: comba_decay_bwd needs the workspace filled by "
                         "comba_decay_fwd_save")
    _memory(workspace, workspace.get_device() == dev)  # (the library checks that it holds the states)
    ws = _workspace(lib.comba_decay_bwd_workspace_bytes, shp, scratch, q.device)
    _run(lib.comba_decay_bwd(shp, *ptrs, *given,
                             *(_ptr(out[n]) for n in ("dq", "dk", "dv", "dg", "dh0")),
                             workspace.data_ptr(), workspace.numel(), ws.data_ptr(), ws.numel(),
                             _on(stream, dev, ws, *out.values())))
    return out


def comba_decay_step(q, k, v, g, state, *, slots=None, scale=None, stream=None):
    """One token per row: returns o [B,H,dv]; ``state`` [S,H,dk,dv] float32 is updated in
    place.  q [B,Hq,dk], k [B,Hk,dk], v [B,Hv,dv], g [B,H] or [H]; slots as in
    comba_conv_step."""
    import torch

    if q.dim() != 3 or state.dim() != 4:
        raise CombaError("comba: q must be [B,heads,dk] and state [S,H,dk,dv]")
    rows, pool = q.shape[0], state.shape[0]
    shp, ptrs, (H, dk, dv), dev = _decay_shape(1, q, k, v, g, scale, rows, 0, None)
    o = _outputs(v, H)
    _run(load_library().comba_decay_step(
        shp, *ptrs, _dense("state", state, (pool, H, dk, dv), torch.float32, dev),
        _slots(slots, rows, dev), pool, o.data_ptr(), _on(stream, dev, o)))
    return o


# ---- norms after and before a block ---------------------------------------------------
def _norm_shape(y, x, weight, post_weight, z, scale, activation, eps, stream_dtype):
    import torch

    code, dev, dt, f32, shape = _code(y, "y"), y.get_device(), y.dtype, torch.float32, y.shape
    lead = len(shape) - 1
    if lead < 0 or shape[-1] < 1:
        raise CombaError("comba: y must be [..,C]")
    if stream_dtype is not dt and stream_dtype is not f32:
        raise CombaError("comba: the stream must be float32 or of y's dtype")
    C = shape[-1]
    shp = _NORM.pack(y.numel() // C, C, code, COMBA_F32 if stream_dtype is f32 else COMBA_BF16,
                     _activation(activation, _NORM_ACT), eps,
                     0 if y.is_contiguous() else _row("y", y, lead, shape, dt, dev),
                     _row("z", z, lead, shape, dt, dev),
                     _row("x", x, lead, shape, stream_dtype, dev))
    ptrs = (y.data_ptr(), _ptr(x), _ptr(z),
            _dense("post_weight", post_weight, (C,), f32, dev),
            _dense("scale", scale, (C,), f32, dev), _dense("weight", weight, (C,), f32, dev))
    return shp, ptrs


def comba_block_norm_fwd(y, x=None, weight=None, *, post_weight=None, z=None, scale=None,
                         activation="silu", eps=1e-6, stream_dtype=None, stream=None):
    """A block's output y [..,C] joins the residual stream x, and the next block's input leaves
    it.  Returns (r, n): with rms(u) = sqrt(mean(u^2) + eps) over the channels,

    p = y / rms(y) post_weight,  r = x + scale p act(z),  n = r / rms(r) weight.

    y, x and z may be column slices; z and n have y's dtype, x and r are float32 or have it too
    (without x: ``stream_dtype``, by default y's).  post_weight, scale and weight are [C] float32;
    each of them, x and z may be None: no norm after the block, a scale of one, no norm before
    the next (n is None), an empty stream, no gate."""
    st = stream_dtype or (y.dtype if x is None else x.dtype)
    shp, ptrs = _norm_shape(y, x, weight, post_weight, z, scale, activation, eps, st)
    r = _like(y, st)
    n = None if weight is None else _like(y)
    _run(load_library().comba_block_norm_fwd(shp, *ptrs, r.data_ptr(), _ptr(n),
                                             _on(stream, y.get_device(), r, n)))
    return r, n


def comba_block_norm_bwd(y, x, weight, dr, dn, *, post_weight=None, z=None, scale=None,
                         activation="silu", eps=1e-6, need_dx=True, stream_dtype=None,
                         workspace=None, stream=None):
    """Backward of comba_block_norm_fwd from dr (the stream's dtype) and dn (y's), either of
    which may be None.  Returns dict dy, dx, dz, dpost_weight, dscale, dweight (None where the
    input is absent)."""
    lib = load_library()
    st = stream_dtype or (dr.dtype if dr is not None else y.dtype if x is None else x.dtype)
    shp, ptrs = _norm_shape(y, x, weight, post_weight, z, scale, activation, eps, st)
    dev = y.get_device()
    grads = (_dense("dr", dr, y.shape, st, dev), _dense("dn", dn, y.shape, y.dtype, dev))
    out = {"dy": _like(y), "dx": _like(y, st) if need_dx and x is not None else None,
           "dz": None if z is None else _like(y),
           "dpost_weight": None if post_weight is None else _like(post_weight),
           "dscale": None if scale is None else _like(scale),
           "dweight": None if weight is None else _like(weight)}
    ws = _workspace(lib.comba_block_norm_workspace_bytes, shp, workspace, y.device)
    _run(lib.comba_block_norm_bwd(shp, *ptrs, *grads, *(_ptr(t) for t in out.values()),
                                  ws.data_ptr(), ws.numel(), _on(stream, dev, ws, *out.values())))
    return out


# ---- torch.autograd ---------------------------------------------------------------
_FNS = {}


def _functions():
    if _FNS:
        return _FNS
    import torch
    from torch.autograd.function import once_differentiable  # the kernels leave no graph

    def needed(ctx, grads):
        return tuple(g if n else None for g, n in zip(grads, ctx.needs_input_grad))

    class Decay(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, g, h0, cu_seqlens, kw, grad):
            ctx.set_materialize_grads(False)
            # (needs_input_grad is set where gradients are off, too)
            if grad and g.dim() == 1 and ctx.needs_input_grad[3]:
                raise CombaError("comba: decays [H] are constants: pass g [B,T,H] to train them")
            if not (grad and any(ctx.needs_input_grad)):  # no backward: no states kept for it
                return comba_decay_fwd(q, k, v, g, h0, cu_seqlens=cu_seqlens, **kw)
            o, ht, ws = comba_decay_fwd_save(q, k, v, g, h0, cu_seqlens=cu_seqlens, **kw)
            ctx.save_for_backward(q, k, v, g, h0, cu_seqlens, ws)
            ctx.kw = kw
            return o, ht

        @staticmethod
        @once_differentiable
        def backward(ctx, do, dht):
            q, k, v, g, h0, cu_seqlens, ws = ctx.saved_tensors
            do = q.new_zeros(q.shape[:2] + (g.shape[-1], v.shape[-1])) if do is None \
                else do.contiguous()
            gr = comba_decay_bwd(q, k, v, g, h0, do, None if dht is None else dht.contiguous(),
                                 workspace=ws, need_dg=ctx.needs_input_grad[3],
                                 need_dh0=h0 is not None and ctx.needs_input_grad[4],
                                 cu_seqlens=cu_seqlens, **ctx.kw)
            names = ("dq", "dk", "dv", "dg", "dh0")
            return needed(ctx, tuple(gr[n] for n in names) + (None, None, None))

    class BlockNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, y, x, weight, post_weight, z, scale, kw):
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(y, x, weight, post_weight, z, scale)
            ctx.kw = kw
            r, n = comba_block_norm_fwd(y, x, weight, post_weight=post_weight, z=z, scale=scale,
                                        **kw)
            ctx.stream_dtype = r.dtype
            return r, n

        @staticmethod
        @once_differentiable
        def backward(ctx, dr, dn):
            y, x, weight, post_weight, z, scale = ctx.saved_tensors
            kw = dict(ctx.kw, stream_dtype=ctx.stream_dtype)
            gr = comba_block_norm_bwd(y, x, weight, None if dr is None else dr.contiguous(),
                                      None if dn is None else dn.contiguous(),
                                      post_weight=post_weight, z=z, scale=scale,
                                      need_dx=ctx.needs_input_grad[1], **kw)
            names = ("dy", "dx", "dweight", "dpost_weight", "dz", "dscale")
            return needed(ctx, tuple(gr[n] for n in names) + (None,))

    _FNS.update(decay=Decay, norm=BlockNorm)
    return _FNS


def comba_decay(q, k, v, g, h0=None, *, scale=None, cu_seqlens=None, cu_seqlens_host=None):
    """Differentiable comba_decay_fwd: (o, ht); gradients flow to q, k, v, h0 and g [B,T,H].
    A call that a backward can follow keeps a state every 64 tokens until it has run."""
    import torch

    kw = dict(scale=scale, cu_seqlens_host=_kept_offsets(cu_seqlens_host))
    return _functions()["decay"].apply(q, k, v, g, h0, cu_seqlens, kw, torch.is_grad_enabled())


def comba_block_norm(y, x=None, weight=None, *, post_weight=None, z=None, scale=None,
                     activation="silu", eps=1e-6, stream_dtype=None):
    """Differentiable comba_block_norm_fwd: (r, n); gradients flow to every tensor."""
    kw = dict(activation=activation, eps=eps, stream_dtype=stream_dtype)
    return _functions()["norm"].apply(y, x, weight, post_weight, z, scale, kw)
