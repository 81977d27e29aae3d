"""GPU parity of the layer's operators (convolution with history, selective scan,
group norm per token) against the fp64 reference in oracle/layer.py.

The kernels compute in fp32 on inputs exact in their storage type, so an fp32
output is held to a norm-wise max relative error of 1e-5 (the repository's bar
for fp32: sums of up to some 1e4 terms with 2^-24 each, in trees or short runs),
and a bf16 output to one unit in its last place, 2^-8 of the value, plus the
same 1e-5 of the tensor's largest."""
import zlib

import numpy as np
import pytest

from comba_inputs import bf16_round
from gpu_helpers import maxrel
from oracle import layer as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _log(msg):
    print(msg, flush=True)


def _dt(name):
    import torch

    return torch.bfloat16 if name == "bf16" else torch.float32


def _dev(x, dtype=None):
    import torch

    return None if x is None else \
        torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype or torch.float32)


def _slice(x, dtype, before=0, after=0):
    """x on the device as a column slice of wider rows."""
    import torch

    if x is None:
        return None
    wide = torch.full(x.shape[:-1] + (before + x.shape[-1] + after,), float("nan"), device="cuda",
                      dtype=dtype)
    wide[..., before:before + x.shape[-1]] = _dev(x, dtype)
    return wide[..., before:before + x.shape[-1]]


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _hold(name, got, want, bf16):
    got = _np(got).reshape(np.shape(want))
    if want.size == 0:
        return
    assert np.all(np.isfinite(got)), name
    if bf16:
        bound = 2.0 ** -8 * np.abs(want) + 1e-5 * np.max(np.abs(want))
        worst = np.max(np.abs(got - want) - bound)
        assert worst <= 0, (name, worst, np.max(np.abs(got - want)))
    else:
        assert maxrel(got, want) <= 1e-5, (name, maxrel(got, want))


def _spans(B, T, lens):
    lens = [T] * B if lens is None else lens
    ends = np.cumsum([0] + list(lens))
    return [(int(a), int(b)) for a, b in zip(ends[:-1], ends[1:])], ends


def _packed(lens, host):
    import torch

    if lens is None:
        return {}
    cu = np.cumsum([0] + list(lens)).astype(np.int32)
    kw = {"cu_seqlens": _dev(cu, torch.int32)}
    if host:
        kw["cu_seqlens_host"] = cu
    return kw


def _rnd(rng, dtype, *shape, scale=1.0):
    x = (scale * rng.standard_normal(shape)).astype(np.float32)
    return bf16_round(x) if dtype == "bf16" else x


# ---- convolution -------------------------------------------------------------
CONV = [
    ("bf16_k4", dict(B=2, T=70, D=64, K=4)),
    ("bf16_k4_wide", dict(B=1, T=133, D=520, K=4, off=8)),
    ("bf16_k3_odd", dict(B=2, T=33, D=37, K=3, off=3)),
    ("bf16_k2_none", dict(B=3, T=5, D=16, K=2, act="none", bias=False)),
    ("bf16_t1", dict(B=4, T=1, D=24, K=4)),
    ("bf16_t2", dict(B=2, T=2, D=8, K=4, dht=True)),
    ("f32_k4", dict(B=2, T=65, D=20, K=4, dtype="f32", off=4)),
    ("f32_k3_odd", dict(B=1, T=40, D=7, K=3, dtype="f32", off=1)),
    ("f32_zero_history", dict(B=2, T=9, D=12, K=4, dtype="f32", h0=False)),
    ("packed", dict(D=72, K=4, lens=[1, 0, 2, 31, 32, 33, 0, 3, 130, 5], host=True, dht=True)),
    ("packed_dev_only", dict(D=40, K=3, lens=[64, 1, 1, 1, 0, 200], dtype="f32")),
    ("packed_odd", dict(D=33, K=4, lens=[2, 2, 2, 2, 2, 2, 60], off=5, dht=True)),
    ("f32_pairs", dict(B=2, T=37, D=22, K=3, dtype="f32", off=2, dht=True)),
    ("bf16_pairs", dict(B=2, T=70, D=50, K=2, off=2, act="none")),
]


def _conv_case(name, B=1, T=0, D=0, K=4, dtype="bf16", act="silu", bias=True, h0=True, dht=False,
               lens=None, off=0, host=False):
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    spans, _ = _spans(B, T, lens)
    n, S = spans[-1][1], len(spans)
    B, T = (B, T) if lens is None else (1, n)
    c = dict(x=_rnd(rng, dtype, n, D), w=_rnd(rng, "f32", D, K, scale=0.5),
             b=_rnd(rng, "f32", D) if bias else None,
             h0=_rnd(rng, dtype, S, K - 1, D) if h0 else None, dy=_rnd(rng, dtype, n, D),
             dht=_rnd(rng, dtype, S, K - 1, D) if dht else None)
    dt = _dt(dtype)
    dev = dict(x=_slice(c["x"].reshape(B, T, D), dt, off, off), w=_dev(c["w"]), b=_dev(c["b"]),
               h0=_dev(c["h0"], dt), dy=_dev(c["dy"].reshape(B, T, D), dt), dht=_dev(c["dht"], dt))
    return c, dev, spans, dict(_packed(lens, host), activation=act), dtype == "bf16"


@pytest.mark.parametrize("name,kw", CONV, ids=[c[0] for c in CONV])
def test_conv_parity(name, kw):
    import paper_2506_02475_amd as comba

    _log("conv " + name)
    c, d, spans, call, bf16 = _conv_case(name, **kw)
    y, ht = comba.comba_conv_fwd(d["x"], d["w"], d["b"], d["h0"], **call)
    gr = comba.comba_conv_bwd(d["x"], d["w"], d["b"], d["h0"], d["dy"], d["dht"], **call)
    act = call["activation"]
    ry, rht = ref.conv_fwd(c["x"], c["w"], c["b"], c["h0"], spans, act)
    rg = ref.conv_bwd(c["x"], c["w"], c["b"], c["h0"], c["dy"], c["dht"], spans, act)
    _hold("y", y, ry, bf16)
    assert np.array_equal(_np(ht), rht)  # copies
    _hold("dx", gr["dx"], rg["dx"], bf16)
    _hold("dh0", gr["dh0"], rg["dh0"], bf16)
    _hold("dw", gr["dw"], rg["dw"], False)
    assert (gr["dbias"] is None) == (c["b"] is None)
    if c["b"] is not None:
        _hold("dbias", gr["dbias"], rg["dbias"], False)


def test_conv_longer_runs():
    # enough tokens that the runs and the workgroups' sums are many
    import paper_2506_02475_amd as comba

    _log("conv long")
    c, d, spans, call, bf16 = _conv_case("long", D=48, K=4, lens=[3000, 1, 0, 1777, 4096], host=True)
    y, _ = comba.comba_conv_fwd(d["x"], d["w"], d["b"], d["h0"], **call)
    gr = comba.comba_conv_bwd(d["x"], d["w"], d["b"], d["h0"], d["dy"], **call)
    _hold("y", y, ref.conv_fwd(c["x"], c["w"], c["b"], c["h0"], spans)[0], bf16)
    rg = ref.conv_bwd(c["x"], c["w"], c["b"], c["h0"], c["dy"], None, spans)
    for n, b in (("dx", bf16), ("dh0", bf16), ("dw", False), ("dbias", False)):
        _hold(n, gr[n], rg[n], b)


@pytest.mark.parametrize("dtype,T,D", [("bf16", 8200, 4100), ("bf16", 8200, 4099),
                                       ("f32", 4110, 4100), ("f32", 4110, 4099)])
def test_conv_large_inputs(dtype, T, D):
    """Beyond 64 MiB of x, checked on some channels (no channel meets another)."""
    import torch

    import paper_2506_02475_amd as comba

    _log("conv large %s %d" % (dtype, D))
    torch.manual_seed(D)
    dt, lens = _dt(dtype), [T - 1300, 1, 0, 1299]
    spans, _ = _spans(1, 0, lens)
    x, dy = (torch.randn(1, T, D, device="cuda").to(dt) for _ in range(2))
    h0, dht = (torch.randn(4, 3, D, device="cuda").to(dt) for _ in range(2))
    w, b = torch.randn(D, 4, device="cuda") * 0.5, torch.randn(D, device="cuda")
    call = _packed(lens, True)
    y, ht = comba.comba_conv_fwd(x, w, b, h0, **call)
    gr = comba.comba_conv_bwd(x, w, b, h0, dy, dht, **call)
    at = [0, 1, 5, 2050, D - 4, D - 3, D - 2, D - 1]
    cx, cdy, ch0, cdht = (_np(t[..., at]) for t in (x[0], dy[0], h0, dht))
    cw, cb = _np(w[at]), _np(b[at])
    ry, rht = ref.conv_fwd(cx, cw, cb, ch0, spans)
    rg = ref.conv_bwd(cx, cw, cb, ch0, cdy, cdht, spans)
    bf16 = dtype == "bf16"
    _hold("y", y[0][:, at], ry, bf16)
    assert np.array_equal(_np(ht[..., at]), rht)
    _hold("dx", gr["dx"][0][:, at], rg["dx"], bf16)
    _hold("dh0", gr["dh0"][..., at], rg["dh0"], bf16)
    _hold("dw", gr["dw"][at], rg["dw"], False)
    _hold("dbias", gr["dbias"][at], rg["dbias"], False)


@pytest.mark.parametrize("dtype,D,K,off", [("bf16", 72, 4, 8), ("bf16", 35, 3, 1), ("f32", 20, 2, 4)])
def test_conv_steps_follow_the_prompt(dtype, D, K, off):
    """Steps through slots of a larger pool, one padding row per step, against the prompt."""
    import torch

    import paper_2506_02475_amd as comba

    _log("conv steps %s %d" % (dtype, D))
    rng = np.random.default_rng(D)
    B, T, S = 3, 6, 7
    dt = _dt(dtype)
    x, w, b = _rnd(rng, dtype, B, T, D), _rnd(rng, "f32", D, K), _rnd(rng, "f32", D)
    h0 = _rnd(rng, dtype, B, K - 1, D)
    pool = _dev(_rnd(rng, dtype, S, K - 1, D), dt)
    before = pool.clone()
    place = [5, 0, 3]
    slots = _dev(np.array([5, -1, 0, 3, S]), torch.int32)
    pool[place] = _dev(h0, dt)
    rows = [0, 2, 3]
    ry, rht = ref.conv_fwd(x.reshape(-1, D), w, b, h0, _spans(B, T, None)[0])
    for t in range(T):
        xs = np.full((5, D), np.nan, np.float32)
        xs[rows] = x[:, t]
        y = comba.comba_conv_step(_slice(xs, dt, off, off), _dev(w), _dev(b), pool, slots=slots)
        _hold("y", y[rows], ry.reshape(B, T, D)[:, t], dtype == "bf16")
        assert not _np(y)[[1, 4]].any()  # padding
    assert np.array_equal(_np(pool)[place], rht)
    rest = [i for i in range(S) if i not in place]
    assert torch.equal(pool[rest], before[rest])


# ---- selective scan -----------------------------------------------------------
SELECT = [
    ("bf16_n16", dict(B=2, T=65, D=64, N=16)),
    ("bf16_n16_t1", dict(B=3, T=1, D=64, N=16)),
    ("bf16_n16_t64", dict(B=1, T=64, D=128, N=16, dht=True)),
    ("bf16_n16_t200", dict(B=1, T=200, D=192, N=16, G=3, dht=True, off=5)),
    ("bf16_n16_odd", dict(B=2, T=77, D=70, N=16, G=2, off=3, dht=True)),
    ("bf16_n8", dict(B=1, T=129, D=130, N=8, off=1, dht=True)),
    ("bf16_n32", dict(B=2, T=96, D=36, N=32, dht=True)),
    ("bf16_n32_odd", dict(B=1, T=70, D=33, N=32, off=7)),
    ("f32_n16", dict(B=2, T=100, D=68, N=16, dtype="f32", dht=True)),
    ("f32_n8_g2", dict(B=1, T=333, D=50, N=8, G=2, dtype="f32", off=1, dht=True)),
    ("f32_n32", dict(B=1, T=130, D=40, N=32, G=2, dtype="f32", off=4)),
    ("bare", dict(B=2, T=40, D=20, N=16, dtype="f32", z=False, skip=False, bias=False, h0=False,
                  softplus=False)),
    ("no_gate", dict(B=1, T=90, D=64, N=16, z=False, dht=True)),
    ("packed", dict(D=64, N=16, lens=[1, 0, 63, 64, 65, 0, 3, 300, 32, 31], host=True, dht=True)),
    ("packed_dev_only", dict(D=24, N=8, lens=[5, 128, 0, 40], dtype="f32", dht=True)),
    ("packed_odd", dict(D=21, N=32, lens=[2, 2, 70, 1], off=1)),
    ("long", dict(B=1, T=3000, D=24, N=16, dtype="f32", dht=True)),
    ("one_channel", dict(B=2, T=37, D=1, N=16, dtype="f32", dht=True)),
]


def _select_case(name, B=1, T=0, D=0, N=16, G=1, dtype="bf16", z=True, skip=True, bias=True, h0=True,
                 dht=False, lens=None, off=0, host=False, softplus=True):
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    spans, _ = _spans(B, T, lens)
    n, S = spans[-1][1], len(spans)
    lead = (B, T) if lens is None else (1, n)
    tau = np.exp(rng.uniform(np.log(1e-3), np.log(0.1), D))
    delta = _rnd(rng, dtype, n, D, scale=0.5)
    if not softplus:
        delta = _rnd(rng, dtype, n, D) ** 2 / 16 if dtype == "f32" else bf16_round(np.abs(delta) / 8)
    c = dict(u=_rnd(rng, dtype, n, D), delta=delta,
             A=(-np.arange(1, N + 1) * np.exp(0.1 * rng.standard_normal((D, N)))).astype(np.float32),
             B=_rnd(rng, dtype, n, G, N), C=_rnd(rng, dtype, n, G, N),
             D=_rnd(rng, "f32", D) if skip else None, z=_rnd(rng, dtype, n, D) if z else None,
             bias=np.log(np.expm1(tau)).astype(np.float32) if bias else None,
             h0=_rnd(rng, "f32", S, D, N) if h0 else None)
    dt = _dt(dtype)

    def rows(x):
        return None if x is None else x.reshape(lead + x.shape[1:])

    d = {k: _dev(c[k]) for k in ("A", "D", "bias", "h0")}
    d["u"], d["delta"] = _dev(rows(c["u"]), dt), _slice(rows(c["delta"]), dt, 0, 2 * off)
    d["z"] = _slice(rows(c["z"]), dt, off, off)
    for k in ("B", "C"):
        d[k] = _slice(rows(c[k].reshape(n, G * N)), dt, off, 0).unflatten(-1, (G, N))
    order = ("u", "delta", "A", "B", "C", "D", "z", "bias", "h0")
    dy = _rnd(rng, dtype, n, D)
    dh = _rnd(rng, "f32", S, D, N) if dht else None
    kw = dict(_packed(lens, host), delta_softplus=softplus)
    return ([c[k] for k in order], [d[k] for k in order], dy, dh, _dev(rows(dy), dt), _dev(dh), spans,
            kw, dtype == "bf16")


def _check_select(name, kw):
    import paper_2506_02475_amd as comba

    host, dev, dy, dht, ddy, ddht, spans, call, bf16 = _select_case(name, **kw)
    sp = call["delta_softplus"]
    y, ht = comba.comba_select_fwd(*dev, **call)
    y2, ht2, ws = comba.comba_select_fwd_save(*dev, **call)
    gr = comba.comba_select_bwd(*dev, ddy, ddht, workspace=ws, **call)
    ry, rht = ref.select_fwd(*host, spans, sp)
    rg = ref.select_bwd(*host, dy, dht, spans, sp)
    for a, b in ((y, ht), (y2, ht2)):
        _hold("y", a, ry, bf16)
        _hold("ht", b, rht, False)
    for n in ("du", "ddelta", "dB", "dC"):
        _hold(n, gr[n], rg[n], bf16)
    _hold("dA", gr["dA"], rg["dA"], False)
    _hold("dh0", gr["dh0"], rg["dh0"], False)
    for n, i, b in (("dz", 6, bf16), ("dD", 5, False), ("ddelta_bias", 7, False)):
        assert (gr[n] is None) == (host[i] is None), n
        if host[i] is not None:
            _hold(n, gr[n], rg[n], b)


@pytest.mark.parametrize("name,kw", SELECT, ids=[c[0] for c in SELECT])
def test_select_parity(name, kw):
    _log("select " + name)
    _check_select(name, kw)


@pytest.mark.parametrize("dtype,D,N,G,off", [("bf16", 64, 16, 1, 0), ("bf16", 70, 16, 2, 3),
                                             ("f32", 33, 8, 1, 1), ("bf16", 100, 32, 1, 4)])
def test_select_steps_follow_the_prompt(dtype, D, N, G, off):
    import torch

    import paper_2506_02475_amd as comba

    _log("select steps %s %d %d" % (dtype, D, N))
    B, T, S = 3, 5, 8
    host, dev, _, _, _, _, spans, _, bf16 = _select_case("steps%d" % D, B=B, T=T, D=D, N=N, G=G,
                                                         dtype=dtype, off=off)
    ry, rht = ref.select_fwd(*host, spans)
    pool = torch.randn(S, D, N, device="cuda")
    before = pool.clone()
    place, rows = [6, 1, 4], [1, 2, 4]
    slots = _dev(np.array([-7, 6, 1, S + 3, 4]), torch.int32)
    pool[place] = dev[8]

    def pad(x, t):  # the step's rows among padding
        if x is None:
            return None
        wide = torch.full((5,) + x.shape[2:], float("nan"), dtype=x.dtype, device="cuda")
        wide[rows] = x[:, t]
        return wide

    u, delta, A, Bm, Cm, skip, z, bias, _ = dev
    for t in range(T):
        y = comba.comba_select_step(pad(u, t), pad(delta, t), A, pad(Bm, t), pad(Cm, t), skip,
                                    pad(z, t), bias, pool, slots=slots)
        _hold("y", y[rows], ry.reshape(B, T, D)[:, t], bf16)
        assert not _np(y)[[0, 3]].any()
    _hold("state", pool[place], rht, False)
    rest = [i for i in range(S) if i not in place]
    assert torch.equal(pool[rest], before[rest])


def test_step_states_beyond_32_bit_offsets():
    """A pool of more than 2^31 state values: the last slot is its own."""
    import torch

    import paper_2506_02475_amd as comba

    D, N = 4096, 16
    S = 2 ** 31 // (D * N) + 3
    _log("pool of %d slots" % S)
    pool = torch.zeros(S, D, N, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    u = torch.randn(2, D, device="cuda", generator=g)
    Bm = torch.randn(2, N, device="cuda", generator=g)
    A = -torch.rand(D, N, device="cuda", generator=g)
    slots = torch.tensor([S - 1, 0], dtype=torch.int32, device="cuda")
    y = comba.comba_select_step(u, u, A, Bm, Bm, None, None, None, pool, slots=slots)
    want = (torch.nn.functional.softplus(u.double()) * u.double())[..., None] * Bm.double()[:, None]
    assert maxrel(_np(pool[[S - 1, 0]]), want.cpu().numpy()) <= 1e-5
    assert maxrel(_np(y), (want * Bm.double()[:, None]).sum(-1).cpu().numpy()) <= 1e-5
    assert not pool[1].any() and not pool[S - 2].any()


# ---- group norm ---------------------------------------------------------------
NORM = [
    ("bf16_128", dict(rows=37, C=512, G=4)),
    ("bf16_gate", dict(rows=130, C=256, G=4, gate=True, off=8)),
    ("bf16_odd", dict(rows=9, C=99, G=3, gate=True, off=3)),
    ("f32_in_bf16_out", dict(rows=65, C=1024, G=4, xt="f32", gate=True, act="sigmoid", off=4)),
    ("f32_small_groups", dict(rows=21, C=60, G=20, dtype="f32")),
    ("f32_single_channels", dict(rows=5, C=6, G=6, dtype="f32", gate=True)),
    ("f32_one_group", dict(rows=11, C=1000, G=1, dtype="f32", act="none", off=1)),
    ("bf16_one_group_1024", dict(rows=6, C=1024, G=1, gate=True)),
    ("bf16_wide", dict(rows=7, C=1501, G=1, gate=True, off=1)),
    ("f32_wide_groups", dict(rows=3, C=5000, G=2, dtype="f32", act="sigmoid")),
    ("bf16_wide_8k", dict(rows=4, C=8192, G=1)),
    ("bf16_one_group_4096", dict(rows=5, C=4096, G=1, gate=True)),
    ("f32_two_groups_3000", dict(rows=700, C=6000, G=2, dtype="f32")),
    ("f32_wide_rows", dict(rows=600, C=4100, G=1, dtype="f32", gate=True)),
    ("bf16_100", dict(rows=50, C=1100, G=11, act="silu")),
    ("no_affine", dict(rows=8, C=256, G=2, affine=False, gate=True)),
    ("one_row", dict(rows=1, C=2048, G=16, xt="f32", gate=True)),
    ("many_rows", dict(rows=9000, C=128, G=2, gate=True)),
    ("bf16_odd_6001", dict(rows=5, C=6001, G=1, gate=True, off=1)),
    ("f32_in_two_groups_8k", dict(rows=270, C=16384, G=2, xt="f32", gate=True)),
    ("bf16_beyond_registers", dict(rows=600, C=9000, G=1, gate=True)),
    ("f32_beyond_registers_odd", dict(rows=5, C=24603, G=3, dtype="f32", gate=True, off=1)),
]


def _norm_case(name, rows=1, C=64, G=1, dtype="bf16", xt=None, act="silu", gate=False, off=0,
               affine=True):
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    xt = xt or dtype
    x = _rnd(rng, xt, rows, C) + (1.0 if xt == "f32" else 0.0)
    w = 1 + _rnd(rng, "f32", C, scale=0.2) if affine else None
    b = _rnd(rng, "f32", C, scale=0.2) if affine else None
    z = _rnd(rng, dtype, rows, C) if gate else None
    dy = _rnd(rng, dtype, rows, C)
    dev = (_slice(x, _dt(xt), off, off), G, _dev(w), _dev(b), _slice(z, _dt(dtype), off, 0))
    return (x, G, w, b, z), dev, dy, _dev(dy, _dt(dtype)), act, xt == "bf16", dtype


@pytest.mark.parametrize("name,kw", NORM, ids=[c[0] for c in NORM])
def test_group_norm_parity(name, kw):
    import paper_2506_02475_amd as comba

    _log("norm " + name)
    host, dev, dy, ddy, act, xb, dtype = _norm_case(name, **kw)
    y = comba.comba_group_norm_fwd(*dev, activation=act, out_dtype=_dt(dtype))
    gr = comba.comba_group_norm_bwd(*dev, ddy, activation=act)
    _hold("y", y, ref.group_norm_fwd(*host, act), dtype == "bf16")
    rg = ref.group_norm_bwd(*host, dy, act)
    _hold("dx", gr["dx"], rg["dx"], xb)
    assert (gr["dz"] is None) == (host[4] is None)
    if host[4] is not None:
        _hold("dz", gr["dz"], rg["dz"], dtype == "bf16")
    for n, i in (("dweight", 2), ("dbias", 3)):
        assert (gr[n] is None) == (host[i] is None)
        if host[i] is not None:
            _hold(n, gr[n], rg[n], False)


# ---- what holds for all of them --------------------------------------------------
def test_autograd_gives_the_direct_calls_gradients():
    import torch

    import paper_2506_02475_amd as comba

    _log("autograd")
    c, d, spans, call, _ = _conv_case("autograd", D=40, K=4, lens=[3, 0, 50], dht=True)
    ins = [d[k].detach().clone().requires_grad_() for k in ("x", "w", "b", "h0")]
    y, ht = comba.comba_conv(*ins, **call)
    got = torch.autograd.grad([y, ht], ins, [d["dy"], d["dht"]])
    gr = comba.comba_conv_bwd(d["x"], d["w"], d["b"], d["h0"], d["dy"], d["dht"], **call)
    for g, n in zip(got, ("dx", "dw", "dbias", "dh0")):
        assert torch.equal(g, gr[n]), n

    host, dev, _, _, ddy, ddht, spans, call, _ = _select_case("autograd", B=2, T=50, D=40, N=16,
                                                             dht=True, off=4)
    ins = [t.detach().requires_grad_() for t in dev]
    y, ht = comba.comba_select(*ins, **call)
    got = torch.autograd.grad([y, ht], ins, [ddy, ddht])
    _, _, ws = comba.comba_select_fwd_save(*dev, **call)
    gr = comba.comba_select_bwd(*dev, ddy, ddht, workspace=ws, **call)
    for g, n in zip(got, ("du", "ddelta", "dA", "dB", "dC", "dD", "dz", "ddelta_bias", "dh0")):
        assert torch.equal(g, gr[n]), n
    # only the final state is used
    y, ht = comba.comba_select(*ins, **call)
    got = torch.autograd.grad(ht, ins[:5], ddht)
    gr = comba.comba_select_bwd(*dev, torch.zeros_like(ddy), ddht, workspace=ws, **call)
    for g, n in zip(got, ("du", "ddelta", "dA", "dB", "dC")):
        assert torch.equal(g, gr[n]), n

    host, dev, dy, ddy, act, _, dtype = _norm_case("autograd", rows=20, C=96, G=3, gate=True)
    ins = [dev[0], dev[2], dev[3], dev[4]]
    ins = [t.detach().requires_grad_() for t in ins]
    y = comba.comba_group_norm(ins[0], 3, *ins[1:])
    got = torch.autograd.grad(y, ins, ddy)
    gr = comba.comba_group_norm_bwd(*dev, ddy)
    for g, n in zip(got, ("dx", "dweight", "dbias", "dz")):
        assert torch.equal(g, gr[n]), n


def test_two_calls_give_the_same_bits():
    import torch

    import paper_2506_02475_amd as comba

    _log("same bits")
    host, dev, _, _, ddy, ddht, _, call, _ = _select_case("bits", D=130, N=16,
                                                         lens=[500, 3, 0, 200], dht=True)

    def once():
        y, ht, ws = comba.comba_select_fwd_save(*dev, **call)
        gr = comba.comba_select_bwd(*dev, ddy, ddht, workspace=ws, **call)
        return [y, ht] + [gr[n] for n in sorted(gr)]

    for a, b in zip(once(), once()):
        assert torch.equal(a, b)


def test_non_finite_values_stay_in_their_sequence():
    """A NaN input and an infinite one reach their own sequence only, and reach it."""
    import torch

    import paper_2506_02475_amd as comba

    _log("non-finite")
    lens = [40, 70, 33, 64]
    host, dev, _, _, ddy, _, spans, call, _ = _select_case("nan", D=24, N=16, lens=lens)
    clean = comba.comba_select_fwd_save(*dev, **call)
    gc = comba.comba_select_bwd(*dev, ddy, workspace=clean[2], **call)
    u = dev[0].clone()
    u[0, 50, 3] = float("nan")      # sequence 1
    u[0, 40 + 70 + 5, 7] = float("inf")  # sequence 2
    bad = [u] + list(dev[1:])
    y, ht, ws = comba.comba_select_fwd_save(*bad, **call)
    gr = comba.comba_select_bwd(*bad, ddy, workspace=ws, **call)
    for a, b in ((0, 40), (143, 207)):
        assert torch.equal(y[:, a:b], clean[0][:, a:b])
        for n in ("du", "ddelta", "dz", "dB", "dC"):
            assert torch.equal(gr[n][:, a:b], gc[n][:, a:b]), n
    assert torch.equal(ht[[0, 3]], clean[1][[0, 3]])
    others = [c for c in range(24) if c != 3]
    assert torch.equal(y[0, 40:110][:, others], clean[0][0, 40:110][:, others])
    assert torch.isnan(ht[1, 3]).all() and torch.isnan(y[0, 50:110, 3]).all()
    assert not torch.isfinite(ht[2, 7]).any()

    c, d, spans, call, _ = _conv_case("nan", D=24, K=4, lens=lens)
    clean = comba.comba_conv_fwd(d["x"], d["w"], d["b"], d["h0"], **call)
    x = d["x"].clone()
    x[0, 109, 2] = float("nan")  # the last token of sequence 1
    y, ht = comba.comba_conv_fwd(x, d["w"], d["b"], d["h0"], **call)
    assert torch.isnan(y[0, 109, 2]) and torch.isnan(ht[1, 2, 2])
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[0, 109, 2] = False
    assert torch.equal(y[keep], clean[0][keep])


def test_calls_without_tokens_pass_the_states_through():
    import torch

    import paper_2506_02475_amd as comba

    _log("no tokens")
    bf = torch.bfloat16
    x = torch.empty(2, 0, 32, device="cuda", dtype=bf)
    w, b = torch.randn(32, 4, device="cuda"), torch.randn(32, device="cuda")
    h = torch.randn(2, 3, 32, device="cuda").to(bf)
    y, ht = comba.comba_conv_fwd(x, w, b, h)
    gr = comba.comba_conv_bwd(x, w, b, h, x, h)
    assert y.shape == x.shape and torch.equal(ht, h) and torch.equal(gr["dh0"], h)
    assert not gr["dw"].any() and not gr["dbias"].any()
    A, s0 = -torch.rand(32, 16, device="cuda"), torch.randn(2, 32, 16, device="cuda")
    bc = torch.empty(2, 0, 1, 16, device="cuda", dtype=bf)
    args = (x, x, A, bc, bc, b, x, b, s0)
    y, ht, ws = comba.comba_select_fwd_save(*args)
    gr = comba.comba_select_bwd(*args, x, s0, workspace=ws)
    assert torch.equal(ht, s0) and torch.equal(gr["dh0"], s0)
    assert not gr["dA"].any() and not gr["dD"].any() and not gr["ddelta_bias"].any()
    e = torch.empty(0, 32, device="cuda", dtype=bf)
    assert comba.comba_group_norm_fwd(e, 2, w[:, 0].contiguous(), b).shape == (0, 32)
    gr = comba.comba_group_norm_bwd(e, 2, w[:, 0].contiguous(), b, None, e)
    assert not gr["dweight"].any() and not gr["dbias"].any()
    e = torch.empty(0, 32, device="cuda", dtype=bf)
    assert comba.comba_conv_step(e, w, b, h).numel() == 0


def test_malformed_device_offsets_stay_in_bounds():
    """Offsets that run backwards or past the tokens (no host copy to check) are clamped on the
    device: the calls end, and what they give is undefined."""
    import torch

    import paper_2506_02475_amd as comba

    _log("malformed offsets")
    host, dev, _, _, ddy, _, _, call, _ = _select_case("malformed", D=24, N=16, lens=[40, 30, 20])
    call["cu_seqlens"] = torch.tensor([-5, 60, 10, 4000], dtype=torch.int32, device="cuda")
    y, ht, ws = comba.comba_select_fwd_save(*dev, **call)
    comba.comba_select_bwd(*dev, ddy, workspace=ws, **call)
    c, d, _, ccall, _ = _conv_case("malformed", D=24, K=4, lens=[40, 30, 20])
    ccall["cu_seqlens"] = call["cu_seqlens"]
    comba.comba_conv_fwd(d["x"], d["w"], d["b"], d["h0"], **ccall)
    comba.comba_conv_bwd(d["x"], d["w"], d["b"], d["h0"], d["dy"], **ccall)
    torch.cuda.synchronize()


def test_another_stream_and_a_graph():
    """On a side stream, and captured in a graph whose replays follow new inputs."""
    import torch

    import paper_2506_02475_amd as comba

    _log("streams and graphs")
    bf = torch.bfloat16
    B, D, N = 4, 256, 16
    x, z = torch.randn(B, D, device="cuda").to(bf), torch.randn(B, D, device="cuda").to(bf)
    w, b = torch.randn(D, 4, device="cuda"), torch.randn(D, device="cuda")
    A, Bm = -torch.rand(D, N, device="cuda"), torch.randn(B, N, device="cuda").to(bf)
    cs, ss = torch.randn(B, 3, D, device="cuda").to(bf), torch.randn(B, D, N, device="cuda")

    def step(cs, ss):
        u = comba.comba_conv_step(x, w, b, cs)
        y = comba.comba_select_step(u, u, A, Bm, Bm, b, None, b, ss)
        return comba.comba_group_norm_fwd(y, 4, b, b, z)

    def eager(n):
        c, s = cs0.clone(), ss0.clone()
        for k in range(n):
            x.copy_(xs[k])
            y = step(c, s)
        return y, c, s

    xs = [torch.randn(B, D, device="cuda").to(bf) for _ in range(4)]
    cs0, ss0 = cs.clone(), ss.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y1 = eager(2)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, c in zip(y1, eager(2)):
        assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cs, ss)
    cs.copy_(cs0)
    ss.copy_(ss0)
    for k in range(4):
        x.copy_(xs[k])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, cs, ss)]
        for a, c in zip(got, eager(k + 1)):
            assert torch.equal(a, c), k


SEGMENTED = [
    ("one_row", dict(B=1, T=1500, D=40, N=16, dht=True)),
    ("one_row_f32", dict(B=1, T=2311, D=12, N=8, dtype="f32", dht=True)),
    ("two_rows_n32", dict(B=2, T=900, D=20, N=32, z=False, dht=True)),
    ("no_states", dict(B=1, T=700, D=33, N=16, h0=False, off=1)),
    ("packed", dict(D=24, N=16, lens=[1100, 1, 0, 64, 700, 129], host=True, dht=True)),
    ("packed_many", dict(D=24, N=16, lens=[7, 60, 0, 33] * 15 + [1300, 5, 0, 900, 200], host=True,
                         dht=True)),
    ("packed_many_f32", dict(D=72, N=8, lens=[1, 0, 2] * 40 + [1000], dtype="f32", host=True,
                             dht=True)),
    ("packed_mixed", dict(D=3000, N=16, lens=[900, 400, 150, 30, 400], z=False, host=True)),
]


@pytest.mark.parametrize("name,kw", SEGMENTED, ids=[c[0] for c in SEGMENTED])
def test_select_rows_cut_into_segments(name, kw):
    """Few long rows: their segments run side by side."""
    _log("select segments " + name)
    _check_select("seg_" + name, kw)


def test_a_stream_given_by_handle():
    """Every call on a stream that is not torch's current one, its temporary memory reused by the
    current stream right after: the results are those of the current stream."""
    import torch

    import paper_2506_02475_amd as comba

    _log("stream handle")
    host, dev, _, _, ddy, _, _, call, _ = _select_case("handle", B=2, T=400, D=96, N=16)
    c, d, _, ccall, _ = _conv_case("handle", B=2, T=300, D=64, K=4)
    _, ndev, _, ndy, act, _, _ = _norm_case("handle", rows=300, C=256, G=2, gate=True)

    def calls(s):
        y, ht, ws = comba.comba_select_fwd_save(*dev, stream=s, **call)
        out = [y, ht]
        gr = comba.comba_select_bwd(*dev, ddy, workspace=ws, stream=s, **call)
        out += [gr[k] for k in sorted(gr)]
        out += list(comba.comba_select_fwd(*dev, stream=s, **call))
        out += list(comba.comba_conv_fwd(d["x"], d["w"], d["b"], d["h0"], stream=s, **ccall))
        gr = comba.comba_conv_bwd(d["x"], d["w"], d["b"], d["h0"], d["dy"], stream=s, **ccall)
        out += [gr[k] for k in sorted(gr)]
        out.append(comba.comba_group_norm_fwd(*ndev, activation=act, stream=s))
        gr = comba.comba_group_norm_bwd(*ndev, ndy, activation=act, stream=s)
        out += [gr[k] for k in sorted(gr)]
        del ws
        for _ in range(8):  # the current stream takes what was freed
            torch.full((1 << 20,), float("nan"), device="cuda")
        return out

    want = calls(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = calls(side.cuda_stream)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def test_values_before_a_nan_are_untouched():
    """A NaN reaches its own channel's later outputs, not the earlier ones of its chunk, tile or
    segment; its gradients not the later tokens'."""
    import torch

    import paper_2506_02475_amd as comba

    _log("before a NaN")
    host, dev, _, _, ddy, _, _, call, _ = _select_case("causal", B=1, T=700, D=40, N=16)
    y0, _, ws = comba.comba_select_fwd_save(*dev, **call)
    g0 = comba.comba_select_bwd(*dev, ddy, workspace=ws, **call)
    for t in (0, 5, 333, 699):
        u = dev[0].clone()
        u[0, t, 7] = float("nan")
        y, _, _ = comba.comba_select_fwd_save(u, *dev[1:], **call)
        assert torch.equal(y[0, :t], y0[0, :t]) and torch.isnan(y[0, t:, 7]).all()
        other = [c for c in range(40) if c != 7]
        assert torch.equal(y[0][:, other], y0[0][:, other])
        dy = ddy.clone()
        dy[0, t, 7] = float("nan")
        g = comba.comba_select_bwd(*dev, dy, workspace=ws, **call)
        for n in ("du", "ddelta"):
            assert torch.equal(g[n][0, t + 1:], g0[n][0, t + 1:]), (t, n)
            assert torch.isnan(g[n][0, :t + 1, 7]).all(), (t, n)
            assert torch.equal(g[n][0][:, other], g0[n][0][:, other]), (t, n)
