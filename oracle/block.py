"""fp64 reference of a block's operators: linear attention with a decay for each head,
the norms after and before a block with gate, residual scale and stream.

TEST INFRASTRUCTURE ONLY: imported by tests/, never by the product path.

Written token by token from the definitions, with the derivatives by hand;
``spans`` lists the sequences' token ranges of the flattened token axis.

    decay   S_t = exp(g_t) S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t
    block   p = y / rms(y) w1,  t = p act(z),  r = x + s t,  n = r / rms(r) w2
"""
from __future__ import annotations

import numpy as np

from oracle.layer import _f8, act


def _heads(x, H):
    """Every head repeated for the state heads that share it: [tokens, H, d]."""
    return np.repeat(x, H // x.shape[1], axis=1)


def _gates(g, n, H):
    return np.broadcast_to(g, (n, H)) if g.ndim == 1 else g


# ---- linear attention with a decay per head ------------------------------------
def decay_fwd(q, k, v, g, h0, scale, spans):
    """q, k [tokens, heads, dk], v [tokens, heads, dv], g [tokens, H] or [H], h0
    [S, H, dk, dv] or None: (o [tokens, H, dv], ht [S, H, dk, dv])."""
    q, k, v, g, h0 = _f8(q, k, v, g, h0)
    n, H = q.shape[0], g.shape[-1]
    g = _gates(g, n, H)
    q, k, v = _heads(q, H), _heads(k, H), _heads(v, H)
    o, ht = np.zeros((n, H, v.shape[2])), np.zeros((len(spans), H, q.shape[2], v.shape[2]))
    for s, (a, b) in enumerate(spans):
        S = np.zeros(ht.shape[1:]) if h0 is None else h0[s].copy()
        for t in range(a, b):
            S = np.exp(g[t])[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            o[t] = scale * np.einsum("hij,hi->hj", S, q[t])
        ht[s] = S
    return o, ht


def decay_bwd(q, k, v, g, h0, do, dht, scale, spans):
    q, k, v, g, h0, do, dht = _f8(q, k, v, g, h0, do, dht)
    n, H = q.shape[0], g.shape[-1]
    heads = (q.shape[1], k.shape[1], v.shape[1])
    g = _gates(g, n, H)
    q, k, v = _heads(q, H), _heads(k, H), _heads(v, H)
    dq, dk, dv, dg = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros((n, H))
    dh0 = np.zeros((len(spans), H, q.shape[2], v.shape[2]))
    for s, (a, b) in enumerate(spans):
        S = [np.zeros(dh0.shape[1:]) if h0 is None else h0[s]]
        for t in range(a, b):
            S.append(np.exp(g[t])[:, None, None] * S[-1] + k[t][:, :, None] * v[t][:, None, :])
        D = np.zeros(dh0.shape[1:]) if dht is None else dht[s].copy()
        for t in range(b - 1, a - 1, -1):
            dq[t] = scale * np.einsum("hij,hj->hi", S[t - a + 1], do[t])
            D = D + scale * q[t][:, :, None] * do[t][:, None, :]
            dk[t] = np.einsum("hij,hj->hi", D, v[t])
            dv[t] = np.einsum("hij,hi->hj", D, k[t])
            dg[t] = np.exp(g[t]) * (D * S[t - a]).sum((1, 2))
            D = np.exp(g[t])[:, None, None] * D
        dh0[s] = D

    def shared(d, m):
        return d.reshape(n, m, H // m, d.shape[2]).sum(2)

    return {"dq": shared(dq, heads[0]), "dk": shared(dk, heads[1]), "dv": shared(dv, heads[2]),
            "dg": dg, "dh0": dh0}


def decay_step(q, k, v, g, state, slots, scale):
    """One token per row: (o [B, H, dv], the pool after it).  Rows whose slot lies outside
    the pool give zeros."""
    q, k, v, g, state = _f8(q, k, v, g, state)
    state = state.copy()
    o = np.zeros((q.shape[0], state.shape[1], v.shape[2]))
    g = _gates(g, q.shape[0], state.shape[1])
    for b, s in enumerate(range(q.shape[0]) if slots is None else slots):
        if 0 <= s < len(state):
            x, h = decay_fwd(q[b:b + 1], k[b:b + 1], v[b:b + 1], g[b:b + 1], state[s:s + 1], scale,
                             [(0, 1)])
            o[b], state[s] = x[0], h[0]
    return o, state


# ---- norms after and before a block ------------------------------------------------
def _rms(x, eps):
    return 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def _back(d, xh, rstd, terms=False):
    """Through xh = x rstd (``terms``: the sum of its terms' absolute values)."""
    if terms:
        return rstd * (np.abs(d) + np.abs(xh) * np.abs(d * xh).mean(-1, keepdims=True))
    return rstd * (d - xh * (d * xh).mean(-1, keepdims=True))


def block_fwd(y, x, z, w1, sc, w2, activation="silu", eps=1e-6):
    """(r, n or None) of rows [rows, C]."""
    y, x, z, w1, sc, w2 = _f8(y, x, z, w1, sc, w2)
    p = y if w1 is None else y * _rms(y, eps) * w1
    t = p if z is None else p * act(activation, z)[0]
    r = t if sc is None else sc * t
    r = r if x is None else x + r
    return r, None if w2 is None else r * _rms(r, eps) * w2


def block_bwd(y, x, z, w1, sc, w2, dr, dn, activation="silu", eps=1e-6, terms=False):
    """``terms``: instead of the gradients, the sums of the absolute values of what is added and
    subtracted for them (a norm of one channel leaves 1e-6 of its gradient's terms)."""
    y, x, z, w1, sc, w2, dr, dn = _f8(y, x, z, w1, sc, w2, dr, dn)
    r1 = None if w1 is None else _rms(y, eps)
    yh = y if w1 is None else y * r1
    p = yh if w1 is None else yh * w1
    gate, slope = (1.0, None) if z is None else act(activation, z)
    t = p * gate
    r = t if sc is None else sc * t
    r = r if x is None else x + r
    d = np.zeros_like(y) if dr is None else dr.copy()
    if terms:
        p, t, r, yh, gate, d = (np.abs(v) for v in (p, t, r, yh, gate, d))
        slope = None if z is None else np.abs(slope)
        w1, sc, w2, dn = (None if v is None else np.abs(v) for v in (w1, sc, w2, dn))
    out = {}
    if w2 is not None:
        r2 = _rms(r, eps)
        dn = np.zeros_like(y) if dn is None else dn
        out["dweight"] = (dn * r * r2).sum(0)
        d = d + _back(dn * w2, r * r2, r2, terms)
    if x is not None:
        out["dx"] = d
    if sc is not None:
        out["dscale"] = (d * t).sum(0)
        d = d * sc
    if z is not None:
        out["dz"] = d * p * slope
        d = d * gate
    if w1 is not None:
        out["dpost_weight"] = (d * yh).sum(0)
        d = _back(d * w1, yh, r1, terms)
    out["dy"] = d
    return out
