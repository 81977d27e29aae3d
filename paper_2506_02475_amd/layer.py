"""The layer's operators around and beside the token mixer (include/comba_layer.h):
the short causal convolution with its history, the selective state space scan and
the group norm per token.

    y, ht = comba_conv_fwd(x, w, bias, h0)              # prompts; comba_conv_step: one token
    y, ht = comba_select_fwd(u, delta, A, B, C, D, z, delta_bias, h0)   # .._step: one token
    y = comba_group_norm_fwd(x, groups, weight, bias, z)

and, differentiable (torch.autograd), comba_conv, comba_select, comba_group_norm.
Activations are bfloat16 or float32 and so are their gradients and outputs;
parameters, their gradients and the scan's states are float32.  Tensors may be
column slices of a wider row (a projection's output) where noted; everything
else is contiguous, on the current device.  Packed sequences pass ``cu_seqlens`` (and, to have the
offsets checked, ``cu_seqlens_host``) as in the package's other calls.
"""
from __future__ import annotations

import ctypes
import struct

from . import (COMBA_BF16, COMBA_F32, CombaError, _check, _host_offsets, _kept_offsets, _ptr,
               load_library)

__all__ = ["comba_conv_fwd", "comba_conv_bwd", "comba_conv_step", "comba_conv",
           "comba_select_fwd", "comba_select_fwd_save", "comba_select_bwd", "comba_select_step",
           "comba_select", "comba_group_norm_fwd", "comba_group_norm_bwd", "comba_group_norm",
           "CombaConvShape", "CombaSelectShape", "CombaGroupNormShape"]

ACTIVATIONS = {None: 0, "none": 0, "silu": 1, "sigmoid": 2}
_I32, _I64, _P = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class CombaConvShape(ctypes.Structure):
    _fields_ = [("B", _I32), ("T", _I32), ("D", _I32), ("K", _I32), ("num_seqs", _I32),
                ("cu_seqlens", _P), ("cu_seqlens_host", _P), ("in_dtype", ctypes.c_int),
                ("activation", ctypes.c_int), ("x_row", _I64)]


class CombaSelectShape(ctypes.Structure):
    _fields_ = [("B", _I32), ("T", _I32), ("D", _I32), ("N", _I32), ("G", _I32),
                ("num_seqs", _I32), ("cu_seqlens", _P), ("cu_seqlens_host", _P),
                ("in_dtype", ctypes.c_int), ("delta_softplus", _I32), ("u_row", _I64),
                ("delta_row", _I64), ("z_row", _I64), ("b_row", _I64), ("c_row", _I64)]


class CombaGroupNormShape(ctypes.Structure):
    _fields_ = [("rows", _I64), ("C", _I32), ("G", _I32), ("x_dtype", ctypes.c_int),
                ("out_dtype", ctypes.c_int), ("activation", ctypes.c_int), ("eps", ctypes.c_float),
                ("x_row", _I64), ("z_row", _I64)]


# A call packs its shape struct with these (a third of the cost of a ctypes
# Structure: at one token per call the binding, not the kernel, bounds the rate).
_CONV = struct.Struct("@iiiiiPPiiq")
_SELECT = struct.Struct("@iiiiiiPPiiqqqqq")
_NORM = struct.Struct("@qiiiiifqq")
assert _CONV.size == ctypes.sizeof(CombaConvShape)
assert _SELECT.size == ctypes.sizeof(CombaSelectShape)
assert _NORM.size == ctypes.sizeof(CombaGroupNormShape)


def bind(lib):
    """Declare the C signatures (called by load_library); the shape structs pass as bytes."""
    P, Z, I = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    for name, args in (("comba_conv_fwd", [P] * 8),
                       ("comba_conv_bwd", [P] * 12 + [Z, P]),
                       ("comba_conv_step", [P] * 6 + [_I32, P, P]),
                       ("comba_select_fwd", [P] * 13 + [Z, P]),
                       ("comba_select_fwd_save", [P] * 13 + [Z, P]),
                       ("comba_select_bwd", [P] * 22 + [Z, P, Z, P]),
                       ("comba_select_step", [P] * 11 + [_I32, P, P]),
                       ("comba_group_norm_fwd", [P] * 7),
                       ("comba_group_norm_bwd", [P] * 11 + [Z, P])):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, I
    for name in ("comba_conv_workspace_bytes", "comba_select_fwd_workspace_bytes",
                 "comba_select_save_bytes", "comba_select_bwd_workspace_bytes",
                 "comba_group_norm_workspace_bytes"):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = [P], Z


def _like(t, dtype=None):
    """An uninitialised contiguous tensor of t's shape (half the host time of new_empty)."""
    import torch

    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


# ---- argument checks -------------------------------------------------------
def _code(t, name):
    if t.get_device() < 0:
        raise CombaError("comba: tensors must be on a GPU device")
    code = _codes().get(t.dtype)
    if code is None:
        raise CombaError("comba: %s must be bfloat16 or float32" % name)
    return code


_CODES = {}


def _codes():
    if not _CODES:
        import torch

        _CODES.update({torch.bfloat16: COMBA_BF16, torch.float32: COMBA_F32})
    return _CODES


def _dense(name, t, shape, dtype, dev):
    """The pointer of a contiguous tensor of this shape (None: absent)."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev \
            or not t.is_contiguous():
        raise CombaError("comba: %s must be a contiguous %s %s on the device"
                         % (name, str(dtype).replace("torch.", ""), list(shape)))
    return t.data_ptr()


_SCAN_ROW = 1 << 22  # the scan's tiles hold rows up to this many elements apart


def _row(name, t, lead, shape, dtype, dev, limit=None):
    """Elements between token rows of ``t`` (``lead`` leading dimensions of tokens,
    then a row): a row's elements are contiguous, the rows evenly spaced and at most
    ``limit`` elements apart."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        raise CombaError("comba: %s must be %s %s on the device"
                         % (name, str(dtype).replace("torch.", ""), list(shape)))
    if t.is_contiguous():
        return 0
    st, n = t.stride(), 1
    if lead == 1 and len(st) == 2 and st[1] == 1 and st[0] >= shape[1]:
        return st[0]
    for d in range(t.dim() - 1, lead - 1, -1):
        if shape[d] != 1 and st[d] != n:
            raise CombaError("comba: a row of %s must be contiguous" % name)
        n *= shape[d]
    row, span = None, 1
    for d in range(lead - 1, -1, -1):
        if shape[d] == 1:
            continue
        if row is None:
            row = st[d]
        elif st[d] != row * span:
            raise CombaError("comba: the rows of %s must be evenly spaced" % name)
        span *= shape[d]
    if row is None:
        return 0
    if row < n:
        raise CombaError("comba: the rows of %s overlap" % name)
    if limit is not None and row > limit:
        raise CombaError("comba: the rows of %s lie %d elements apart, at most %d are supported: "
                         "pass a contiguous copy" % (name, row, limit))
    return row


def _seqs(B, cu_seqlens, cu_seqlens_host, dev):
    """(sequences, device pointer, host offsets) of a call."""
    if cu_seqlens is None:
        if cu_seqlens_host is not None:
            raise CombaError("comba: cu_seqlens_host needs cu_seqlens")
        return B, 0, None
    import torch

    if cu_seqlens.dtype is not torch.int32 or not cu_seqlens.is_contiguous() \
            or cu_seqlens.get_device() != dev or B != 1:
        raise CombaError("comba: cu_seqlens must be contiguous int32 on the device, B == 1")
    N = cu_seqlens.numel() - 1
    return N, cu_seqlens.data_ptr(), _host_offsets(cu_seqlens_host, N + 1)


def _slots(slots, rows, dev):
    if slots is None:
        return None
    import torch

    if slots.dtype is not torch.int32 or slots.shape != (rows,) \
            or not slots.is_contiguous() or slots.get_device() != dev:
        raise CombaError("comba: slots must be contiguous int32 [B] on the device")
    return slots.data_ptr()


def _activation(name, allowed):
    if name not in allowed:
        raise CombaError("comba: activation must be one of %s" % (allowed,))
    return ACTIVATIONS[name]


def _memory(given, here):
    """A caller's workspace: as many bytes as elements, at least, ``here`` on the device."""
    if not here or not given.is_contiguous():
        raise CombaError("comba: a workspace must be contiguous memory on the tensors' device")
    return given


def _workspace(fn, shp, given, device):
    import torch

    nbytes = fn(shp)
    if nbytes == 0:
        _check(2)
    if given is not None and _memory(given, given.device == device).numel() >= nbytes:
        return given
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _host_ptr(host):
    return 0 if host is None else host.ctypes.data


def _run(status):
    if status:
        _check(status)


def _on(stream, dev, *made):
    """The stream handle of a call.  Tensors that the call makes on another stream than
    torch's current one: that stream first waits for the current one, whose work may still
    use the memory that they were given, and they are marked as used there, so that it is
    not given away while the kernels still run."""
    import torch

    cuda = torch._C
    if cuda._cuda_getDevice() != dev:
        raise CombaError("comba: the tensors are on device %d: make it the current device "
                         "(torch.cuda.device)" % dev)
    here = cuda._cuda_getCurrentRawStream(dev)
    if stream is None or stream == here:
        return here
    # (an ExternalStream of handle 0, the default stream, would be another stream)
    ext = torch.cuda.ExternalStream(stream, device=dev) if stream \
        else torch.cuda.default_stream(dev)
    ext.wait_stream(torch.cuda.current_stream(dev))
    for t in made:
        if t is not None:
            t.record_stream(ext)
    return stream


# ---- short causal convolution -------------------------------------------------
_CONV_ACT = (None, "none", "silu")


def _conv_shape(x, w, bias, h0, activation, cu_seqlens, cu_seqlens_host):
    import torch

    code, dev = _code(x, "x"), x.get_device()
    if x.dim() != 3 or w.dim() != 2 or w.shape[0] != x.shape[2]:
        raise CombaError("comba: x must be [B,T,D] and w [D,K]")
    shape = x.shape
    B, T, D = shape
    K = w.shape[1]
    N, cu, host = _seqs(B, cu_seqlens, cu_seqlens_host, dev)
    row = 0 if x.is_contiguous() else _row("x", x, 2, shape, x.dtype, dev)
    shp = _CONV.pack(B, T, D, K, N, cu, _host_ptr(host), code, _activation(activation, _CONV_ACT),
                     row)
    ptrs = (x.data_ptr(), _dense("w", w, (D, K), torch.float32, dev),
            _dense("bias", bias, (D,), torch.float32, dev),
            _dense("h0", h0, (N, K - 1, D), x.dtype, dev))
    return shp, host, ptrs, (N, K - 1, D), dev


def comba_conv_fwd(x, w, bias=None, h0=None, *, activation="silu", cu_seqlens=None,
                   cu_seqlens_host=None, output_final_state=True, stream=None):
    """Short causal depthwise convolution.  Returns (y [B,T,D], ht [N,K-1,D] or None).

    x [B,T,D] (may be a column slice); w [D,K] float32, K = 2..4, the newest token
    under the last tap; bias [D] float32; h0 [N,K-1,D]: each sequence's inputs
    before its first token, oldest first (None: zeros); ht: those before its next."""
    shp, _host, ptrs, state, dev = _conv_shape(x, w, bias, h0, activation, cu_seqlens,
                                               cu_seqlens_host)
    y = _like(x)
    ht = x.new_empty(state) if output_final_state else None
    _run(load_library().comba_conv_fwd(shp, *ptrs, y.data_ptr(), _ptr(ht),
                                       _on(stream, dev, y, ht)))
    return y, ht


def comba_conv_bwd(x, w, bias, h0, dy, dht=None, *, activation="silu", cu_seqlens=None,
                   cu_seqlens_host=None, need_dh0=True, workspace=None, stream=None):
    """Backward of comba_conv_fwd from dy [B,T,D] (and dht [N,K-1,D]), both in the dtype of
    x.  Returns dict dx (dtype of x), dw, dbias (float32; None without bias), dh0."""
    import torch

    lib = load_library()
    shp, _host, ptrs, state, dev = _conv_shape(x, w, bias, h0, activation, cu_seqlens,
                                               cu_seqlens_host)
    grads = (_dense("dy", dy, x.shape, x.dtype, dev), _dense("dht", dht, state, x.dtype, dev))
    out = {"dx": _like(x), "dw": torch.empty_like(w),
           "dbias": None if bias is None else torch.empty_like(bias),
           "dh0": x.new_empty(state) if need_dh0 else None}
    ws = _workspace(lib.comba_conv_workspace_bytes, shp, workspace, x.device)
    _run(lib.comba_conv_bwd(shp, *ptrs, *grads, _ptr(out["dx"]), _ptr(out["dw"]),
                            _ptr(out["dbias"]), _ptr(out["dh0"]), _ptr(ws), ws.numel(),
                            _on(stream, dev, ws, *out.values())))
    return out


def comba_conv_step(x, w, bias, state, *, slots=None, activation="silu", stream=None):
    """One token per row: returns y [B,D]; ``state`` [S,K-1,D] is updated in place.

    x [B,D] (may be a column slice).  Row b uses slot slots[b] (int32 on the device; a
    slot outside [0, S) marks padding: y zero, no state touched), or slot b."""
    import torch

    code, dev, shape, taps, pool = _code(x, "x"), x.get_device(), x.shape, w.shape, state.shape
    if len(shape) != 2 or len(taps) != 2 or taps[0] != shape[1] or len(pool) != 3:
        raise CombaError("comba: x must be [B,D], w [D,K] and state [S,K-1,D]")
    B, D = shape
    K, dt, f32 = taps[1], x.dtype, torch.float32
    shp = _CONV.pack(B, 1, D, K, B, 0, 0, code, _activation(activation, _CONV_ACT),
                     0 if x.is_contiguous() else _row("x", x, 1, shape, dt, dev))
    y = _like(x)
    _run(load_library().comba_conv_step(
        shp, x.data_ptr(), _dense("w", w, taps, f32, dev), _dense("bias", bias, (D,), f32, dev),
        _dense("state", state, (pool[0], K - 1, D), dt, dev), _slots(slots, B, dev), pool[0],
        y.data_ptr(), _on(stream, dev, y)))
    return y


# ---- selective state space scan --------------------------------------------------
def _select_shape(lead, u, delta, A, B, C, D, z, delta_bias, delta_softplus, N, cu, host):
    import torch

    code, dev, dt = _code(u, "u"), u.get_device(), u.dtype
    f32 = torch.float32
    shape, ashape, bshape = u.shape, A.shape, B.shape
    width = shape[-1]
    if len(ashape) != 2 or ashape[0] != width:
        raise CombaError("comba: A must be [D,N]")
    n = ashape[1]
    if len(bshape) == lead + 2:
        G = bshape[lead]
        want = shape[:-1] + (G, n)
    elif len(bshape) == lead + 1:
        G = 1
        want = shape[:-1] + (n,)
    else:
        raise CombaError("comba: B and C must be [..,G,N] or [..,N]")
    if lead == 1:
        batch, T, far = shape[0], 1, None
    else:
        batch, T, far = shape[0], shape[1], _SCAN_ROW
    shp = _SELECT.pack(batch, T, width, n, G, N, cu, _host_ptr(host), code,
                       1 if delta_softplus else 0,
                       0 if u.is_contiguous() else _row("u", u, lead, shape, dt, dev, far),
                       _row("delta", delta, lead, shape, dt, dev, far),
                       _row("z", z, lead, shape, dt, dev, far),
                       _row("B", B, lead, want, dt, dev, far),
                       _row("C", C, lead, want, dt, dev, far))
    ptrs = (u.data_ptr(), delta.data_ptr(), _dense("A", A, ashape, f32, dev), B.data_ptr(),
            C.data_ptr(), _dense("D", D, (width,), f32, dev), None if z is None else z.data_ptr(),
            _dense("delta_bias", delta_bias, (width,), f32, dev))
    return shp, ptrs, n, want


def _select(save, u, delta, A, B, C, D, z, delta_bias, h0, delta_softplus, cu_seqlens,
            cu_seqlens_host, output_final_state, workspace, stream):
    import torch

    lib = load_library()
    _code(u, "u")
    if u.dim() != 3:
        raise CombaError("comba: u must be [B,T,D]")
    S, cu, host = _seqs(u.shape[0], cu_seqlens, cu_seqlens_host, u.get_device())
    shp, ptrs, n, _ = _select_shape(2, u, delta, A, B, C, D, z, delta_bias, delta_softplus, S, cu,
                                    host)
    state = (S, u.shape[2], n)
    h0p = _dense("h0", h0, state, torch.float32, u.get_device())
    y = _like(u)
    ht = A.new_empty(state) if output_final_state else None
    size = lib.comba_select_save_bytes if save else lib.comba_select_fwd_workspace_bytes
    ws = _workspace(size, shp, workspace, u.device)
    fn = lib.comba_select_fwd_save if save else lib.comba_select_fwd
    _run(fn(shp, *ptrs, h0p, y.data_ptr(), _ptr(ht), ws.data_ptr(), ws.numel(),
            _on(stream, u.get_device(), y, ht, ws)))
    return y, ht, ws


def comba_select_fwd(u, delta, A, B, C, D=None, z=None, delta_bias=None, h0=None, *,
                     delta_softplus=True, cu_seqlens=None, cu_seqlens_host=None,
                     output_final_state=True, workspace=None, stream=None):
    """Selective state space scan.  Returns (y [B,T,D], ht [S,D,N] float32 or None).

    With dt = softplus(delta + delta_bias) per channel and token,
    h_t = exp(dt A) h_{t-1} + dt u_t B_t,  y_t = (<C_t, h_t> + D u_t) silu(z_t).
    u, delta, z [B,T,D]; B, C [B,T,G,N] or [B,T,N] (G groups of channels), all of one dtype
    and each possibly a column slice; A [D,N], D, delta_bias [D], h0 [S,D,N] float32.
    D, z, delta_bias and h0 may be None.  N: 8, 16 or 32.  Rows of a slice lie at most 2^22
    elements apart."""
    y, ht, _ = _select(False, u, delta, A, B, C, D, z, delta_bias, h0, delta_softplus, cu_seqlens,
                       cu_seqlens_host, output_final_state, workspace, stream)
    return y, ht


def comba_select_fwd_save(u, delta, A, B, C, D=None, z=None, delta_bias=None, h0=None, *,
                          delta_softplus=True, cu_seqlens=None, cu_seqlens_host=None,
                          output_final_state=True, workspace=None, stream=None):
    """comba_select_fwd that also keeps the states its backward needs.  Returns (y, ht,
    workspace); pass the same inputs and ``workspace`` to comba_select_bwd."""
    return _select(True, u, delta, A, B, C, D, z, delta_bias, h0, delta_softplus, cu_seqlens,
                   cu_seqlens_host, output_final_state, workspace, stream)


def comba_select_bwd(u, delta, A, B, C, D, z, delta_bias, h0, dy, dht=None, *, workspace,
                     delta_softplus=True, cu_seqlens=None, cu_seqlens_host=None, need_dh0=True,
                     scratch=None, stream=None):
    """Backward of comba_select_fwd_save from dy [B,T,D] (dtype of u) and dht [S,D,N] float32,
    with the ``workspace`` it filled; ``scratch``: memory for the call itself, made if absent.
    Returns dict du, ddelta, dz, dB, dC (dtype of u), dA, dD, ddelta_bias, dh0 (float32); the
    entries of absent inputs are None."""
    import torch

    lib = load_library()
    _code(u, "u")
    if u.dim() != 3:
        raise CombaError("comba: u must be [B,T,D]")
    dev, f32 = u.get_device(), torch.float32
    S, cu, host = _seqs(u.shape[0], cu_seqlens, cu_seqlens_host, dev)
    shp, ptrs, n, bshape = _select_shape(2, u, delta, A, B, C, D, z, delta_bias, delta_softplus, S,
                                         cu, host)
    state = (S, u.shape[2], n)
    given = (_dense("h0", h0, state, f32, dev), _dense("dy", dy, u.shape, u.dtype, dev),
             _dense("dht", dht, state, f32, dev))
    out = {"du": _like(u), "ddelta": _like(u),
           "dA": _like(A), "dB": _like(B), "dC": _like(C),
           "dD": None if D is None else _like(D),
           "dz": None if z is None else _like(u),
           "ddelta_bias": None if delta_bias is None else _like(delta_bias),
           "dh0": A.new_empty(state) if need_dh0 else None}
    if workspace is None or _memory(workspace, workspace.get_device() == dev).numel() \
            < lib.comba_select_save_bytes(shp):
        raise CombaError("comba: comba_select_bwd needs the workspace filled by "
                         "comba_select_fwd_save")
    ws = _workspace(lib.comba_select_bwd_workspace_bytes, shp, scratch, u.device)
    _run(lib.comba_select_bwd(
        shp, *ptrs, *given, *(_ptr(out[k]) for k in ("du", "ddelta", "dA", "dB", "dC", "dD", "dz",
                                                     "ddelta_bias", "dh0")),
        workspace.data_ptr(), workspace.numel(), ws.data_ptr(), ws.numel(),
        _on(stream, dev, ws, *out.values())))
    return out


def comba_select_step(u, delta, A, B, C, D, z, delta_bias, state, *, slots=None,
                      delta_softplus=True, stream=None):
    """One token per row: returns y [B,D]; ``state`` [S,D,N] float32 is updated in place.
    u, delta, z [B,D]; B, C [B,G,N] or [B,N]; slots as in comba_conv_step."""
    import torch

    shape, pool = u.shape, state.shape
    if len(shape) != 2 or len(pool) != 3:
        raise CombaError("comba: u must be [B,D] and state [S,D,N]")
    rows = shape[0]
    shp, ptrs, n, _ = _select_shape(1, u, delta, A, B, C, D, z, delta_bias, delta_softplus, rows,
                                    0, None)
    dev = u.get_device()
    y = _like(u)
    _run(load_library().comba_select_step(
        shp, *ptrs, _dense("state", state, (pool[0], shape[1], n), torch.float32, dev),
        _slots(slots, rows, dev), pool[0], y.data_ptr(), _on(stream, dev, y)))
    return y


# ---- group norm per token -------------------------------------------------------
_NORM_ACT = (None, "none", "silu", "sigmoid")


def _norm_shape(x, groups, weight, bias, z, activation, eps, out):
    import torch

    xc, dev, dt, f32, shape = _code(x, "x"), x.get_device(), x.dtype, torch.float32, x.shape
    lead = len(shape) - 1
    if lead < 0 or groups < 1 or shape[-1] < 1 or shape[-1] % groups:
        raise CombaError("comba: x must be [..,C] with C a multiple of groups")
    if out is not torch.bfloat16 and out is not f32:
        raise CombaError("comba: out_dtype must be bfloat16 or float32")
    if out is not dt and dt is not f32:
        raise CombaError("comba: x must be float32 or have the output's dtype")
    C = shape[-1]
    shp = _NORM.pack(x.numel() // C, C, groups, xc,
                     COMBA_BF16 if out is torch.bfloat16 else COMBA_F32,
                     _activation(activation, _NORM_ACT), eps,
                     0 if x.is_contiguous() else _row("x", x, lead, shape, dt, dev),
                     _row("z", z, lead, shape, out, dev))
    ptrs = (x.data_ptr(), _dense("weight", weight, (C,), f32, dev),
            _dense("bias", bias, (C,), f32, dev), None if z is None else z.data_ptr())
    return shp, ptrs


def comba_group_norm_fwd(x, groups, weight=None, bias=None, z=None, *, activation="silu",
                         eps=1e-5, out_dtype=None, stream=None):
    """Group norm of every token over the channels of each of ``groups`` groups, then
    y = act(n), or with the gate z: y = n act(z).

    x [..,C] and z may be column slices; weight, bias [C] float32 or None.  y has
    ``out_dtype`` (default: the dtype of z, else of x); x is float32 or of that dtype."""
    out = out_dtype or (x.dtype if z is None else z.dtype)
    shp, ptrs = _norm_shape(x, groups, weight, bias, z, activation, eps, out)
    y = _like(x, out)
    _run(load_library().comba_group_norm_fwd(shp, *ptrs, y.data_ptr(),
                                             _on(stream, x.get_device(), y)))
    return y


def comba_group_norm_bwd(x, groups, weight, bias, z, dy, *, activation="silu", eps=1e-5,
                         workspace=None, stream=None):
    """Backward of comba_group_norm_fwd from dy (the forward's output dtype).  Returns dict dx
    (dtype of x), dz (dtype of dy, None without z), dweight, dbias (float32, None where absent)."""
    lib = load_library()
    shp, ptrs = _norm_shape(x, groups, weight, bias, z, activation, eps, dy.dtype)
    dyp = _dense("dy", dy, x.shape, dy.dtype, x.get_device())
    out = {"dx": _like(x), "dz": None if z is None else _like(dy),
           "dweight": None if weight is None else _like(weight),
           "dbias": None if bias is None else _like(bias)}
    ws = _workspace(lib.comba_group_norm_workspace_bytes, shp, workspace, x.device)
    _run(lib.comba_group_norm_bwd(shp, *ptrs, dyp, _ptr(out["dx"]), _ptr(out["dz"]),
                                  _ptr(out["dweight"]), _ptr(out["dbias"]), ws.data_ptr(),
                                  ws.numel(), _on(stream, x.get_device(), ws, *out.values())))
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

    class Conv(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, bias, h0, cu_seqlens, kw):
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(x, w, bias, h0, cu_seqlens)
            ctx.kw = kw
            return comba_conv_fwd(x, w, bias, h0, cu_seqlens=cu_seqlens, **kw)

        @staticmethod
        @once_differentiable
        def backward(ctx, dy, dht):
            x, w, bias, h0, cu_seqlens = ctx.saved_tensors
            dy = torch.zeros_like(x, memory_format=torch.contiguous_format) if dy is None \
                else dy.contiguous()
            gr = comba_conv_bwd(x, w, bias, h0, dy, None if dht is None else dht.contiguous(),
                                need_dh0=h0 is not None and ctx.needs_input_grad[3],
                                cu_seqlens=cu_seqlens, **ctx.kw)
            return needed(ctx, (gr["dx"], gr["dw"], gr["dbias"], gr["dh0"], None, None))

    class Select(torch.autograd.Function):
        @staticmethod
        def forward(ctx, u, delta, A, B, C, D, z, bias, h0, cu_seqlens, kw, grad):
            ctx.set_materialize_grads(False)
            if not (grad and any(ctx.needs_input_grad)):  # no backward: no states kept for it
                return comba_select_fwd(u, delta, A, B, C, D, z, bias, h0, cu_seqlens=cu_seqlens,
                                        **kw)
            y, ht, ws = comba_select_fwd_save(u, delta, A, B, C, D, z, bias, h0,
                                              cu_seqlens=cu_seqlens, **kw)
            ctx.save_for_backward(u, delta, A, B, C, D, z, bias, h0, cu_seqlens, ws)
            ctx.kw = kw
            return y, ht

        @staticmethod
        @once_differentiable
        def backward(ctx, dy, dht):
            u, delta, A, B, C, D, z, bias, h0, cu_seqlens, ws = ctx.saved_tensors
            dy = torch.zeros_like(u, memory_format=torch.contiguous_format) if dy is None \
                else dy.contiguous()
            gr = comba_select_bwd(u, delta, A, B, C, D, z, bias, h0, dy,
                                  None if dht is None else dht.contiguous(), workspace=ws,
                                  need_dh0=h0 is not None and ctx.needs_input_grad[8],
                                  cu_seqlens=cu_seqlens, **ctx.kw)
            names = ("du", "ddelta", "dA", "dB", "dC", "dD", "dz", "ddelta_bias", "dh0")
            return needed(ctx, tuple(gr[n] for n in names) + (None, None, None))

    class GroupNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, z, groups, kw, out_dtype):
            ctx.save_for_backward(x, weight, bias, z)
            ctx.groups, ctx.kw = groups, kw
            return comba_group_norm_fwd(x, groups, weight, bias, z, out_dtype=out_dtype, **kw)

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            x, weight, bias, z = ctx.saved_tensors
            gr = comba_group_norm_bwd(x, ctx.groups, weight, bias, z, dy.contiguous(), **ctx.kw)
            return needed(ctx, (gr["dx"], gr["dweight"], gr["dbias"], gr["dz"], None, None, None))

    _FNS.update(conv=Conv, select=Select, norm=GroupNorm)
    return _FNS


def comba_conv(x, w, bias=None, h0=None, *, activation="silu", cu_seqlens=None,
               cu_seqlens_host=None):
    """Differentiable comba_conv_fwd: (y, ht); gradients flow to x, w, bias and h0."""
    kw = dict(activation=activation, cu_seqlens_host=_kept_offsets(cu_seqlens_host))
    return _functions()["conv"].apply(x, w, bias, h0, cu_seqlens, kw)


def comba_select(u, delta, A, B, C, D=None, z=None, delta_bias=None, h0=None, *,
                 delta_softplus=True, cu_seqlens=None, cu_seqlens_host=None):
    """Differentiable comba_select_fwd: (y, ht); gradients flow to every tensor.  A call
    that a backward can follow keeps a state every 48 tokens (N = 8: 32) until it has run."""
    kw = dict(delta_softplus=delta_softplus, cu_seqlens_host=_kept_offsets(cu_seqlens_host))
    import torch

    return _functions()["select"].apply(u, delta, A, B, C, D, z, delta_bias, h0, cu_seqlens, kw,
                                        torch.is_grad_enabled())


def comba_group_norm(x, groups, weight=None, bias=None, z=None, *, activation="silu", eps=1e-5,
                     out_dtype=None):
    """Differentiable comba_group_norm_fwd: gradients flow to x, weight, bias and z."""
    kw = dict(activation=activation, eps=eps)
    return _functions()["norm"].apply(x, weight, bias, z, groups, kw, out_dtype)
