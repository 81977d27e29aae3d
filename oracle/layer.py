"""fp64 reference of the layer's operators: the short causal convolution with its
history, the selective state space scan, the group norm per token.

TEST INFRASTRUCTURE ONLY: imported by tests/, never by the product path.

Written token by token from the definitions, with the derivatives by hand;
``spans`` lists the sequences' token ranges of the flattened token axis.

    conv    xt = [h0; x],  u_t = b + sum_j w_j xt_{t+j},  y = act(u),  ht = last K - 1 rows of xt
    select  dt = softplus(delta + bias),  h_t = exp(dt_t A) h_{t-1} + dt_t u_t B_t,
            s_t = <C_t, h_t> + D u_t,  y = s silu(z)
    norm    n = (x - mean) / sqrt(var + eps) w + b per token and group,  y = act(n) | n act(z)
"""
from __future__ import annotations

import numpy as np


def _sig(x):
    return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))),
                    np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


def _f8(*xs):
    return [None if x is None else np.asarray(x, np.float64) for x in xs]


def act(name, t):
    """(act(t), act'(t))."""
    if name in (None, "none"):
        return t, np.ones_like(t)
    s = _sig(t)
    if name == "silu":
        return t * s, s + t * s * (1.0 - s)
    return s, s * (1.0 - s)


# ---- convolution -------------------------------------------------------------
def conv_fwd(x, w, b, h0, spans, activation="silu"):
    """x [tokens, D], w [D, K], h0 [S, K-1, D]: (y [tokens, D], ht [S, K-1, D])."""
    x, w, b, h0 = _f8(x, w, b, h0)
    D, K = w.shape
    y, ht = np.zeros_like(x), np.zeros((len(spans), K - 1, D))
    for s, (p, q) in enumerate(spans):
        xt = np.concatenate([np.zeros((K - 1, D)) if h0 is None else h0[s], x[p:q]])
        for t in range(q - p):
            u = sum(w[:, j] * xt[t + j] for j in range(K)) + (0.0 if b is None else b)
            y[p + t] = act(activation, u)[0]
        ht[s] = xt[q - p:]
    return y, ht


def conv_bwd(x, w, b, h0, dy, dht, spans, activation="silu"):
    x, w, b, h0, dy, dht = _f8(x, w, b, h0, dy, dht)
    D, K = w.shape
    dx, dw, db = np.zeros_like(x), np.zeros_like(w), np.zeros(D)
    dh0 = np.zeros((len(spans), K - 1, D))
    for s, (p, q) in enumerate(spans):
        n = q - p
        xt = np.concatenate([np.zeros((K - 1, D)) if h0 is None else h0[s], x[p:q]])
        dxt = np.zeros_like(xt)
        if dht is not None:
            dxt[n:] += dht[s]
        for t in range(n):
            u = sum(w[:, j] * xt[t + j] for j in range(K)) + (0.0 if b is None else b)
            du = dy[p + t] * act(activation, u)[1]
            for j in range(K):
                dxt[t + j] += w[:, j] * du
                dw[:, j] += du * xt[t + j]
            db += du
        dx[p:q] = dxt[K - 1:]
        dh0[s] = dxt[:K - 1]
    return {"dx": dx, "dw": dw, "dbias": db, "dh0": dh0}


# ---- selective scan -----------------------------------------------------------
def _wide(x, D):
    """A group's row [G, N] for each of its D / G channels."""
    return np.repeat(x, D // x.shape[0], axis=0)


def _steps(delta, bias, softplus):
    raw = delta + (0.0 if bias is None else bias)
    if not softplus:
        return raw, np.ones_like(raw)
    return np.logaddexp(0.0, raw), _sig(raw)


def select_fwd(u, delta, A, B, C, D, z, bias, h0, spans, softplus=True, keep=False):
    """u, delta, z [tokens, D]; B, C [tokens, G, N]; h0 [S, D, N]: (y, ht), and with
    ``keep`` also every token's state and ungated output."""
    u, delta, A, B, C, D, z, bias, h0 = _f8(u, delta, A, B, C, D, z, bias, h0)
    width, N = A.shape
    dt, _ = _steps(delta, bias, softplus)
    pre, hs = np.zeros_like(u), np.zeros(u.shape + (N,))
    ht = np.zeros((len(spans), width, N)) if h0 is None else h0.copy()
    for s, (p, q) in enumerate(spans):
        h = ht[s]
        for t in range(p, q):
            h = np.exp(dt[t][:, None] * A) * h + (dt[t] * u[t])[:, None] * _wide(B[t], width)
            hs[t] = h
            pre[t] = np.sum(_wide(C[t], width) * h, -1) + (0.0 if D is None else D * u[t])
        ht[s] = h
    y = pre if z is None else pre * act("silu", z)[0]
    return (y, ht, hs, pre) if keep else (y, ht)


def select_bwd(u, delta, A, B, C, D, z, bias, h0, dy, dht, spans, softplus=True):
    _, _, hs, pre = select_fwd(u, delta, A, B, C, D, z, bias, h0, spans, softplus, keep=True)
    u, delta, A, B, C, D, z, bias, h0, dy, dht = _f8(u, delta, A, B, C, D, z, bias, h0, dy, dht)
    width, N = A.shape
    G = B.shape[1]
    dt, slope = _steps(delta, bias, softplus)
    gy, dz = dy, None
    if z is not None:
        a, sl = act("silu", z)
        gy, dz = dy * a, dy * pre * sl
    du, ddelta = np.zeros_like(u), np.zeros_like(u)
    dA, dB, dC = np.zeros_like(A), np.zeros_like(B), np.zeros_like(C)
    dh0 = np.zeros((len(spans), width, N))
    for s, (p, q) in enumerate(spans):
        carry = np.zeros((width, N)) if dht is None else dht[s].copy()
        for t in range(q - 1, p - 1, -1):
            Bw, Cw = _wide(B[t], width), _wide(C[t], width)
            dh = carry + Cw * gy[t][:, None]
            decay = np.exp(dt[t][:, None] * A)
            before = hs[t - 1] if t > p else (np.zeros((width, N)) if h0 is None else h0[s])
            g = dh * decay * before
            gb = np.sum(dh * Bw, -1)
            du[t] = dt[t] * gb + (0.0 if D is None else D * gy[t])
            ddelta[t] = (np.sum(A * g, -1) + u[t] * gb) * slope[t]
            dA += dt[t][:, None] * g
            dB[t] = np.sum((dh * (dt[t] * u[t])[:, None]).reshape(G, -1, N), 1)
            dC[t] = np.sum((hs[t] * gy[t][:, None]).reshape(G, -1, N), 1)
            carry = decay * dh
        dh0[s] = carry
    return {"du": du, "ddelta": ddelta, "dA": dA, "dB": dB, "dC": dC, "dz": dz,
            "dD": np.sum(gy * u, 0), "ddelta_bias": np.sum(ddelta, 0), "dh0": dh0}


# ---- group norm per token ---------------------------------------------------------
def group_norm_fwd(x, groups, w, b, z, activation="silu", eps=1e-5, keep=False):
    """x, z [rows, C]: y [rows, C]."""
    x, w, b, z = _f8(x, w, b, z)
    xg = x.reshape(x.shape[0], groups, -1)
    c = xg - xg.mean(-1, keepdims=True)
    sd = np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    xh = (c / sd).reshape(x.shape)
    n = xh * (1.0 if w is None else w) + (0.0 if b is None else b)
    y = act(activation, n)[0] if z is None else n * act(activation, z)[0]
    return (y, xh, n, sd) if keep else y


def group_norm_bwd(x, groups, w, b, z, dy, activation="silu", eps=1e-5):
    _, xh, n, sd = group_norm_fwd(x, groups, w, b, z, activation, eps, keep=True)
    w, z, dy = _f8(w, z, dy)
    dz = None
    if z is None:
        dn = dy * act(activation, n)[1]
    else:
        a, sl = act(activation, z)
        dn, dz = dy * a, dy * n * sl
    g = (dn * (1.0 if w is None else w)).reshape(len(xh), groups, -1)
    xr = xh.reshape(g.shape)
    dx = (g - g.mean(-1, keepdims=True) - xr * (g * xr).mean(-1, keepdims=True)) / sd
    return {"dx": dx.reshape(xh.shape), "dz": dz, "dweight": np.sum(dn * xh, 0),
            "dbias": np.sum(dn, 0)}
