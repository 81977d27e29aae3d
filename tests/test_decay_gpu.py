"""GPU parity of linear attention with a decay per head against the fp64 reference in
oracle/block.py: rows, packed sequences, shared heads, odd sizes, slices, single tokens."""
import zlib

import numpy as np
import pytest

from block_helpers import column_slice, dev, dt, hold, host, packed, rnd, spans
from oracle import block as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


CASES = [
    ("t1", dict(B=2, T=1, H=2, dk=64, dv=64)),
    ("t2_no_state", dict(B=1, T=2, H=1, dk=64, dv=64, h0=False)),
    ("chunk", dict(B=1, T=64, H=2, dk=64, dv=64)),
    ("chunk_less_one", dict(B=1, T=63, H=2, dk=128, dv=64)),
    ("chunk_and_one", dict(B=2, T=65, H=2, dk=64, dv=128, dht=True)),
    ("d128", dict(B=2, T=200, H=3, dk=128, dv=128, dht=True)),
    ("d256", dict(B=1, T=140, H=2, dk=256, dv=256, dht=True)),
    ("dk256_dv64", dict(B=1, T=70, H=1, dk=256, dv=64, off=8)),
    ("odd_sizes", dict(B=2, T=77, H=2, dk=37, dv=33, off=3, dht=True)),
    ("one_by_one", dict(B=1, T=130, H=2, dk=1, dv=1)),
    ("eights", dict(B=1, T=100, H=2, dk=48, dv=80, off=16)),
    ("eights_unaligned", dict(B=1, T=100, H=2, dk=48, dv=80, off=5)),
    ("dv_200", dict(B=1, T=66, H=2, dk=96, dv=200)),
    ("shared_qk", dict(B=2, T=90, H=6, heads=(2, 3, 6), dk=64, dv=64, dht=True)),
    ("shared_kv", dict(B=1, T=90, H=4, heads=(4, 1, 2), dk=48, dv=40)),
    ("shared_all", dict(B=1, T=70, H=4, heads=(1, 1, 1), dk=32, dv=32, off=1)),
    ("gate_head", dict(B=2, T=130, H=3, dk=64, dv=64, gate="head", dht=True)),
    ("gate_f32", dict(B=1, T=130, H=3, dk=64, dv=64, gate="f32")),
    ("strong_decay", dict(B=1, T=150, H=2, dk=64, dv=64, tau=0.3)),
    ("growth", dict(B=1, T=100, H=2, dk=64, dv=64, tau=-200.0)),
    ("no_decay", dict(B=1, T=200, H=2, dk=64, dv=64, tau=1e9)),
    ("resets", dict(B=1, T=200, H=2, dk=64, dv=64, reset=True, dht=True)),
    ("packed", dict(H=2, dk=64, dv=64, lens=[1, 0, 2, 63, 64, 65, 0, 3, 130, 5], dht=True)),
    ("packed_dev_only", dict(H=3, dk=128, dv=64, lens=[64, 1, 1, 1, 0, 200], host=False)),
    ("packed_odd", dict(H=2, dk=20, dv=50, lens=[2, 2, 2, 70, 0], off=5)),
    ("packed_empty", dict(H=2, dk=64, dv=64, lens=[0, 0, 0], dht=True)),
    ("rows_empty", dict(B=2, T=0, H=2, dk=64, dv=64, dht=True)),
    ("segments", dict(B=1, T=1300, H=1, dk=64, dv=64, dht=True, tau=300.0)),
    ("segments_packed", dict(H=1, dk=64, dv=64, lens=[5, 700, 0, 900, 300], dht=True, tau=300.0)),
    ("segments_no_state", dict(B=2, T=600, H=1, dk=128, dv=32, h0=False, tau=300.0)),
    ("segments_no_state_cut", dict(B=2, T=700, H=1, dk=128, dv=32, h0=False, tau=300.0)),
    ("segments_d256", dict(B=1, T=900, H=1, dk=256, dv=200, dht=True, tau=300.0)),
    ("segments_odd", dict(H=2, dk=33, dv=17, lens=[650, 1, 999], off=1, dht=True, tau=300.0)),
    ("f32_d100_d200", dict(B=1, T=100, H=2, dk=100, dv=200, dtype="f32", dht=True)),
    ("f32_wide_odd", dict(B=1, T=70, H=2, dk=201, dv=130, dtype="f32", off=1, dht=True)),
    ("f32", dict(B=2, T=150, H=2, dk=64, dv=64, dtype="f32", dht=True)),
    ("f32_d128", dict(B=1, T=90, H=2, dk=128, dv=128, dtype="f32")),
    ("f32_d256", dict(B=1, T=70, H=1, dk=256, dv=256, dtype="f32")),
    ("f32_odd", dict(B=1, T=77, H=3, heads=(3, 1, 3), dk=37, dv=33, dtype="f32", off=1, dht=True)),
    ("f32_strong", dict(B=1, T=150, H=2, dk=32, dv=32, dtype="f32", tau=0.3)),
    ("f32_resets", dict(B=1, T=200, H=2, dk=32, dv=32, dtype="f32", reset=True)),
    ("f32_segments", dict(H=1, dk=64, dv=64, lens=[700, 5, 600], dtype="f32", tau=300.0, dht=True)),
]


def _case(name, B=1, T=0, H=1, heads=None, dk=64, dv=64, dtype="bf16", gate="token", h0=True,
          dht=False, lens=None, off=0, host=True, tau=20.0, reset=False):
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    sp = spans(B, T, lens)
    n, S = (B * T if lens is None else sum(lens)), len(sp)
    Hq, Hk, Hv = heads or (H, H, H)
    c = {"q": rnd(rng, dtype, n, Hq, dk, scale=dk ** -0.5),
         "k": rnd(rng, dtype, n, Hk, dk, scale=dk ** -0.5), "v": rnd(rng, dtype, n, Hv, dv)}
    gd = "f32" if gate != "token" or dtype == "f32" else "bf16"
    g = -np.exp(0.5 * rng.standard_normal((H,) if gate == "head" else (n, H))) / tau
    if reset:
        g[rng.random(g.shape) < 0.1] = -np.inf
    c["g"] = rnd(rng, gd, 0) if g.size == 0 and gate != "head" else g.astype(np.float32)
    c["g"] = c["g"].reshape(g.shape)
    if gd == "bf16":
        from comba_inputs import bf16_round

        c["g"] = np.where(np.isfinite(c["g"]), bf16_round(np.where(np.isfinite(c["g"]), c["g"], 0)),
                          c["g"]).astype(np.float32)
    c["h0"] = rnd(rng, "f32", S, H, dk, dv, scale=0.3) if h0 else None
    c["do"] = rnd(rng, dtype, n, H, dv)
    c["dht"] = rnd(rng, "f32", S, H, dk, dv, scale=0.3) if dht else None
    c.update(spans=sp, lens=lens, lead=(1, n) if lens is not None else (B, T), dtype=dtype, gd=gd,
             off=off, host=host, scale=0.7)
    return c


def _inputs(c):
    lead = c["lead"]

    def put(name, lead_dims=2):
        x = c[name].reshape(lead + c[name].shape[1:])
        return column_slice(x, dt(c["dtype"]), 2, c["off"], c["off"]) if c["off"] else \
            dev(x, dt(c["dtype"]))

    q, k, v = put("q"), put("k"), put("v")
    if c["g"].ndim == 1:
        g = dev(c["g"])
    else:
        g = c["g"].reshape(lead + c["g"].shape[1:])
        g = column_slice(g, dt(c["gd"]), 2, c["off"], c["off"]) if c["off"] else dev(g, dt(c["gd"]))
    return q, k, v, g, dev(c["h0"])


def _abs(c):
    a = dict(c)
    for n in ("q", "k", "v", "h0", "do", "dht"):
        a[n] = None if c[n] is None else np.abs(c[n])
    return a


def _fwd(c):
    return ref.decay_fwd(c["q"], c["k"], c["v"], c["g"], c["h0"], c["scale"], c["spans"])


def _bwd(c):
    return ref.decay_bwd(c["q"], c["k"], c["v"], c["g"], c["h0"], c["do"], c["dht"], c["scale"],
                         c["spans"])


@pytest.mark.parametrize("name,kw", CASES, ids=[c[0] for c in CASES])
def test_forward(name, kw):
    import paper_2506_02475_amd as comba

    c = _case(name, **kw)
    o, ht = comba.comba_decay_fwd(*_inputs(c), scale=c["scale"], **packed(c["lens"], c["host"]))
    want, want_t = _fwd(c)
    mag, _ = _fwd(_abs(c))
    hold("o", o, want, mag, c["dtype"])
    hold("ht", ht, want_t, None, "f32")


@pytest.mark.parametrize("name,kw", CASES, ids=[c[0] for c in CASES])
def test_backward(name, kw):
    import paper_2506_02475_amd as comba

    c = _case(name, **kw)
    args, kws = _inputs(c), dict(scale=c["scale"], **packed(c["lens"], c["host"]))
    o, ht, ws = comba.comba_decay_fwd_save(*args, **kws)
    o2, ht2 = comba.comba_decay_fwd(*args, **kws)
    assert bool((o == o2).all()) and bool((ht == ht2).all())
    do = dev(c["do"], dt(c["dtype"])).reshape(c["lead"] + c["do"].shape[1:])
    got = comba.comba_decay_bwd(*args, do, dev(c["dht"]), workspace=ws, **kws)
    want, mag = _bwd(c), _bwd(_abs(c))
    for n in ("dq", "dk", "dv"):
        hold(n, got[n], want[n], mag[n], c["dtype"])
    if c["g"].ndim == 1:
        assert got["dg"] is None
    else:
        # (a pair across the chunk's both ends multiplies two rounded states)
        hold("dg", got["dg"], want["dg"], mag["dg"], c["dtype"], inner=2)
    hold("dh0", got["dh0"], want["dh0"], None, "f32")


@pytest.mark.parametrize("dk", [64, 128, 256])
def test_kept_states_with_columns_of_unlike_size(dk):
    """Values of every second column smaller by 2^12 and keys by 2^8 (queries larger by it) share
    the scale of a block of a kept state.  Its fp16 keeps 11 bits down to 2^-29 of the largest
    value: an eighth of a half step of bf16 more in each term, also for the smaller columns, held
    to their own size; what is below adds 2^-39 of the largest, 2^-19 of a term here."""
    import paper_2506_02475_amd as comba

    c = _case("unlike%d" % dk, B=1, T=200, H=2, dk=dk, dv=64)
    small_v, small_k = np.arange(64) % 2 == 1, np.arange(dk) % 2 == 1
    c["v"] = c["v"] * np.where(small_v, np.float32(2.0 ** -12), np.float32(1))
    c["k"] = c["k"] * np.where(small_k, np.float32(2.0 ** -8), np.float32(1))
    c["q"] = c["q"] * np.where(small_k, np.float32(2.0 ** 8), np.float32(1))
    c["h0"] = (c["h0"] * np.where(small_k, 2.0 ** -8, 1)[:, None]
               * np.where(small_v, 2.0 ** -12, 1)).astype(np.float32)
    o, _ = comba.comba_decay_fwd(*_inputs(c), scale=c["scale"])
    want, mag = _fwd(c)[0], _fwd(_abs(c))[0]
    o = o.reshape(want.shape)
    for m in (small_v, ~small_v):
        hold("o", o[..., np.flatnonzero(m)], want[..., m], 1.125 * mag[..., m], "bf16")


STEPS = [
    ("one", dict(B=1, H=2, dk=64, dv=64)),
    ("slots", dict(B=5, H=3, dk=128, dv=128, pool=9)),
    ("many", dict(B=300, H=4, dk=64, dv=128, pool=301)),
    ("padding", dict(B=6, H=2, dk=64, dv=64, pool=7, pad=True)),
    ("shared", dict(B=3, H=6, heads=(3, 2, 1), dk=48, dv=80, pool=3)),
    ("odd", dict(B=3, H=2, dk=37, dv=33, pool=4, off=3)),
    ("wide", dict(B=2, H=1, dk=256, dv=256, pool=2)),
    ("one_by_one", dict(B=2, H=1, dk=1, dv=1, pool=2)),
    ("gate_head", dict(B=3, H=2, dk=64, dv=64, pool=3, gate="head")),
    ("reset", dict(B=3, H=2, dk=64, dv=64, pool=3, reset=True)),
    ("f32", dict(B=4, H=2, dk=100, dv=100, pool=5, dtype="f32")),
]


@pytest.mark.parametrize("name,kw", STEPS, ids=[c[0] for c in STEPS])
def test_step(name, kw):
    import torch

    import paper_2506_02475_amd as comba

    kw = dict(kw)
    pool, pad = kw.pop("pool", None), kw.pop("pad", False)
    c = _case("step_" + name, T=1, **kw)
    B = kw["B"]
    rng = np.random.default_rng(7)
    slots = None if pool is None else rng.permutation(pool)[:B].astype(np.int32)
    if pad:
        slots[1], slots[3] = -1, pool
    state = rnd(rng, "f32", pool or B, kw["H"], kw["dk"], kw["dv"], scale=0.3)
    q, k, v, g, _ = _inputs(c)
    q, k, v = q[:, 0], k[:, 0], v[:, 0]
    g = g if g.dim() == 1 else g[:, 0]
    st = dev(state)
    o = comba.comba_decay_step(q, k, v, g, st, scale=c["scale"],
                               slots=None if slots is None else dev(slots, torch.int32))
    want, pool_after = ref.decay_step(c["q"], c["k"], c["v"], c["g"], state, slots, c["scale"])
    a = _abs(c)
    mag, _ = ref.decay_step(a["q"], a["k"], a["v"], a["g"], np.abs(state), slots, c["scale"])
    hold("o", o, want, mag, c["dtype"], inner=0)
    hold("state", st, pool_after, None, "f32")
    if pad:
        assert not host(o)[[1, 3]].any()
    rest = [s for s in range(len(state)) if slots is not None and s not in slots]
    assert np.array_equal(host(st)[rest].astype(np.float32), state[rest])
