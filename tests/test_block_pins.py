"""The fp64 reference of a block's operators (oracle/block.py) against what does not share
its code: closed forms, splitting a sequence, and central differences (CPU)."""
import numpy as np
import pytest

from oracle import block as ref
from oracle import step_fwd


def _rng(seed):
    return np.random.default_rng(seed)


def _differences(f, args, grads, seed):
    """Directional central differences along a random direction per input.  Step 1e-5: the
    third-derivative term is about 1e-10, rounding 1e-16 / 1e-5 = 1e-11 of the value, each times
    the sums' size of some 1e2 to 1e3."""
    rng = _rng(seed)
    for i, g in enumerate(grads):
        if g is None or args[i] is None:
            continue
        d, e = rng.standard_normal(np.shape(args[i])), 1e-5
        up, dn = list(args), list(args)
        up[i], dn[i] = args[i] + e * d, args[i] - e * d
        num = (f(*up) - f(*dn)) / (2 * e)
        assert abs(num - float(np.sum(g * d))) <= 1e-6 * (1.0 + abs(num)), (i, num)


@pytest.mark.parametrize("heads", [(4, 4, 4), (2, 1, 4)])
def test_decay_gradients_by_differences(heads):
    rng = _rng(1)
    spans, n, H, dk, dv = [(0, 5), (5, 5), (5, 6), (6, 9)], 9, 4, 3, 2
    q, k, v = (rng.standard_normal((n, h, d)) for h, d in zip(heads, (dk, dk, dv)))
    g, h0 = -rng.random((n, H)), rng.standard_normal((4, H, dk, dv))
    do, dht = rng.standard_normal((n, H, dv)), rng.standard_normal((4, H, dk, dv))

    def loss(q, k, v, g, h0):
        o, ht = ref.decay_fwd(q, k, v, g, h0, 0.7, spans)
        return float(np.sum(do * o) + np.sum(dht * ht))

    gr = ref.decay_bwd(q, k, v, g, h0, do, dht, 0.7, spans)
    _differences(loss, [q, k, v, g, h0], [gr[x] for x in ("dq", "dk", "dv", "dg", "dh0")], 2)


def test_decay_closed_forms():
    rng = _rng(3)
    n, H, d = 7, 2, 3
    q, k, v = (rng.standard_normal((n, H, d)) for _ in range(3))
    # no decay: a masked product; a decay of zero: a token sees itself alone
    o, _ = ref.decay_fwd(q, k, v, np.zeros((n, H)), None, 1.0, [(0, n)])
    P = np.tril(np.einsum("rhd,jhd->hrj", q, k))
    np.testing.assert_allclose(o, np.einsum("hrj,jhd->rhd", P, v), rtol=1e-12, atol=1e-12)
    o, _ = ref.decay_fwd(q, k, v, np.full((n, H), -np.inf), None, 1.0, [(0, n)])
    np.testing.assert_allclose(o, (q * k).sum(-1, keepdims=True) * v, rtol=1e-12, atol=1e-12)
    # constants of the heads are the same for every token
    g = -rng.random(H)
    a, b = (ref.decay_fwd(q, k, v, x, None, 0.5, [(0, n)]) for x in (g, np.tile(g, (n, 1))))
    np.testing.assert_array_equal(a[0], b[0])
    # splitting a sequence
    for cut in (1, 4):
        x, h = ref.decay_fwd(q[:cut], k[:cut], v[:cut], g, None, 0.5, [(0, cut)])
        y, h = ref.decay_fwd(q[cut:], k[cut:], v[cut:], g, h, 0.5, [(0, n - cut)])
        np.testing.assert_allclose(np.concatenate([x, y]), a[0], rtol=1e-13, atol=1e-13)
        np.testing.assert_allclose(h, a[1], rtol=1e-13, atol=1e-13)


def test_decay_is_the_bilinear_recurrence_without_feedback():
    """beta = 1, beta~ = 0, d = 0 in the mixer's own reference."""
    rng = _rng(4)
    B, T, H, d = 2, 9, 2, 64
    q, k, v = (rng.standard_normal((B, T, H, d)).astype(np.float32) for _ in range(3))
    g = -rng.random((B, T, H)).astype(np.float32)
    one, zero = np.ones((B, T, H), np.float32), np.zeros((B, T, H), np.float32)
    o, ht = step_fwd(q, k, v, g, one, np.zeros(H, np.float32), None, beta_tilde=zero)
    mine, st = ref.decay_fwd(*(x.reshape((B * T,) + x.shape[2:]) for x in (q, k, v, g)), None, 1.0,
                             [(0, T), (T, 2 * T)])
    np.testing.assert_allclose(mine.reshape(o.shape), o, rtol=1e-9, atol=1e-9)
    np.testing.assert_allclose(st, ht, rtol=1e-9, atol=1e-9)


@pytest.mark.parametrize("given", ["yxzwsv", "yzwsv", "yxwsv", "yxzsv", "yxzwv", "yxzws", "yv"])
def test_block_gradients_by_differences(given):
    rng = _rng(5)
    rows, C = 3, 6
    full = {"y": rng.standard_normal((rows, C)), "x": rng.standard_normal((rows, C)),
            "z": rng.standard_normal((rows, C)), "w": rng.standard_normal(C),
            "s": rng.standard_normal(C), "v": rng.standard_normal(C)}
    args = [full[c] if c in given else None for c in "yxzwsv"]
    dr, dn = rng.standard_normal((rows, C)), rng.standard_normal((rows, C))

    def loss(*a):
        r, n = ref.block_fwd(*a)
        return float(np.sum(dr * r) + (0.0 if n is None else np.sum(dn * n)))

    g = ref.block_bwd(*args, dr, dn if args[5] is not None else None)
    names = ("dy", "dx", "dz", "dpost_weight", "dscale", "dweight")
    assert set(g) == {n for n, a in zip(names, args) if a is not None}
    _differences(loss, args, [g.get(n) for n in names], 6)
    terms = ref.block_bwd(*args, dr, dn if args[5] is not None else None, terms=True)
    for n in g:
        assert np.all(np.abs(g[n]) <= terms[n] * (1 + 1e-12)) or n in ("dpost_weight", "dscale",
                                                                      "dweight"), n


def test_block_closed_forms():
    rng = _rng(7)
    y, w = rng.standard_normal((4, 5)), rng.standard_normal(5)
    r, n = ref.block_fwd(y, None, None, None, None, None)
    assert n is None and np.array_equal(r, y)
    _, n = ref.block_fwd(3.0 * y, None, None, None, None, w, eps=0.0)
    np.testing.assert_allclose((n / w * n / w).mean(-1), 1.0, rtol=1e-12)
    np.testing.assert_allclose(n, ref.block_fwd(y, None, None, None, None, w, eps=0.0)[1], rtol=1e-12)
