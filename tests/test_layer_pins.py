"""The fp64 reference of the layer's operators (oracle/layer.py) against what does
not share its code: closed forms, numpy's convolution, splitting a sequence, and
central differences for every gradient (CPU)."""
import numpy as np
import pytest

from oracle import layer as ref


def _rng(seed):
    return np.random.default_rng(seed)


def _differences(f, args, names, grads, seed, tol=2e-7):
    """Directional central differences of f(*args) along a random direction per input.
    Step 1e-5: the third-derivative term is about 1e-10, rounding 1e-16 / 1e-5 = 1e-11 of
    the value, each times the sums' size of some 1e2."""
    rng = _rng(seed)
    for i, name in enumerate(names):
        if name is None or args[i] is None:
            continue
        d = rng.standard_normal(np.shape(args[i]))
        e = 1e-5
        up, dn = list(args), list(args)
        up[i], dn[i] = args[i] + e * d, args[i] - e * d
        num = (f(*up) - f(*dn)) / (2 * e)
        ana = float(np.sum(grads[name] * d))
        assert abs(num - ana) <= tol * (1.0 + abs(num)) * 10, (name, num, ana)


@pytest.mark.parametrize("K,act,bias,h0", [(4, "silu", True, True), (2, "none", False, False),
                                           (3, "silu", True, True)])
def test_conv_gradients_by_differences(K, act, bias, h0):
    rng = _rng(K)
    spans, D = [(0, 5), (5, 5), (5, 6), (6, 8)], 3
    x, w = rng.standard_normal((8, D)), rng.standard_normal((D, K))
    b = rng.standard_normal(D) if bias else None
    h = rng.standard_normal((4, K - 1, D)) if h0 else None
    dy, dht = rng.standard_normal((8, D)), rng.standard_normal((4, K - 1, D))

    def loss(x, w, b, h):
        y, ht = ref.conv_fwd(x, w, b, h, spans, act)
        return float(np.sum(dy * y) + np.sum(dht * ht))

    g = ref.conv_bwd(x, w, b, h, dy, dht, spans, act)
    _differences(loss, [x, w, b, h], ["dx", "dw", "dbias", "dh0"], g, 7)


def test_conv_is_numpys_convolution_and_splits():
    rng = _rng(1)
    T, D, K = 17, 2, 4
    x, w = rng.standard_normal((T, D)), rng.standard_normal((D, K))
    y, _ = ref.conv_fwd(x, w, None, None, [(0, T)], "none")
    for c in range(D):
        np.testing.assert_allclose(y[:, c], np.convolve(x[:, c], w[c, ::-1])[:T], rtol=1e-12,
                                   atol=1e-12)
    for cut in (1, 2, 9):
        a, h = ref.conv_fwd(x[:cut], w, None, None, [(0, cut)], "none")
        b, _ = ref.conv_fwd(x[cut:], w, None, h, [(0, T - cut)], "none")
        np.testing.assert_allclose(np.concatenate([a, b]), y, rtol=1e-13, atol=1e-13)


def _select_inputs(seed, T=7, D=4, N=3, G=2, S=3):
    rng = _rng(seed)
    n = rng.standard_normal
    return dict(u=n((T, D)), delta=n((T, D)), A=-np.exp(n((D, N))), B=n((T, G, N)), C=n((T, G, N)),
                D=n(D), z=n((T, D)), bias=n(D), h0=n((S, D, N)), dy=n((T, D)), dht=n((S, D, N)))


@pytest.mark.parametrize("softplus,absent", [(True, ()), (False, ("z", "D", "bias", "h0")),
                                             (True, ("z",))])
def test_select_gradients_by_differences(softplus, absent):
    s = _select_inputs(3)
    for n in absent:
        s[n] = None
    spans = [(0, 4), (4, 4), (4, 7)]
    names = ["u", "delta", "A", "B", "C", "D", "z", "bias", "h0"]

    def loss(*a):
        y, ht = ref.select_fwd(*a, spans, softplus)
        return float(np.sum(s["dy"] * y) + np.sum(s["dht"] * ht))

    g = ref.select_bwd(*[s[n] for n in names], s["dy"], s["dht"], spans, softplus)
    g["dbias"] = g.pop("ddelta_bias")
    _differences(loss, [s[n] for n in names], ["d" + n for n in names], g, 11)


def test_select_closed_form_and_splits():
    # constant step, input and rows: h_t is a geometric series
    T, D, N = 9, 2, 3
    A = -np.array([[0.5, 1.0, 2.0], [0.1, 0.2, 0.3]])
    one = np.ones
    dt = 0.3
    y, ht = ref.select_fwd(one((T, D)), dt * one((T, D)), A, one((T, 1, N)), one((T, 1, N)), None,
                           None, None, None, [(0, T)], softplus=False)
    r = np.exp(dt * A)
    for t in range(T):
        np.testing.assert_allclose(y[t], np.sum(dt * (1 - r ** (t + 1)) / (1 - r), -1), rtol=1e-12)
    s = _select_inputs(5, T=11, S=1)
    full, hfull = ref.select_fwd(s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"],
                                 s["bias"], s["h0"], [(0, 11)])
    a, h = ref.select_fwd(s["u"][:4], s["delta"][:4], s["A"], s["B"][:4], s["C"][:4], s["D"],
                          s["z"][:4], s["bias"], s["h0"], [(0, 4)])
    b, h = ref.select_fwd(s["u"][4:], s["delta"][4:], s["A"], s["B"][4:], s["C"][4:], s["D"],
                          s["z"][4:], s["bias"], h, [(0, 7)])
    np.testing.assert_allclose(np.concatenate([a, b]), full, rtol=1e-12)
    np.testing.assert_allclose(h, hfull, rtol=1e-12)


@pytest.mark.parametrize("act", ["none", "silu", "sigmoid"])
@pytest.mark.parametrize("gate", [False, True])
def test_group_norm_gradients_by_differences(act, gate):
    rng = _rng(13)
    x, w, b = rng.standard_normal((3, 10)), rng.standard_normal(10), rng.standard_normal(10)
    z = rng.standard_normal((3, 10)) if gate else None
    dy = rng.standard_normal((3, 10))
    g = ref.group_norm_bwd(x, 2, w, b, z, dy, act)

    def loss(x, w, b, z):
        return float(np.sum(dy * ref.group_norm_fwd(x, 2, w, b, z, act)))

    _differences(loss, [x, w, b, z], ["dx", "dweight", "dbias", "dz"], g, 17)


def test_group_norm_rows_are_normal_and_shift_free():
    rng = _rng(19)
    x = rng.standard_normal((4, 24))
    y = ref.group_norm_fwd(x, 3, None, None, None, "none", eps=0.0).reshape(4, 3, 8)
    np.testing.assert_allclose(y.mean(-1), 0.0, atol=1e-14)
    np.testing.assert_allclose((y * y).mean(-1), 1.0, rtol=1e-13)
    again = ref.group_norm_fwd(5.0 * x + 3.0, 3, None, None, None, "none", eps=0.0)
    np.testing.assert_allclose(again.reshape(4, 3, 8), y, atol=1e-12)
