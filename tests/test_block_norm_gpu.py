"""GPU parity of the norms after and before a block (gate, residual scale, stream) against
the fp64 reference in oracle/block.py."""
import zlib

import numpy as np
import pytest

from block_helpers import HALF, column_slice, dev, dt, host, rnd
from oracle import block as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


CASES = [
    ("one_row", dict(rows=1, C=64)),
    ("one_channel", dict(rows=5, C=1)),
    ("c256", dict(rows=9, C=256)),
    ("c500", dict(rows=700, C=500)),
    ("c1000", dict(rows=70, C=1000, off=4)),
    ("c2048", dict(rows=300, C=2048)),
    ("c4096", dict(rows=600, C=4096)),
    ("c8192", dict(rows=20, C=8192)),
    ("c8200_wide", dict(rows=7, C=8200)),
    ("c9001_wide", dict(rows=300, C=9001)),
    ("c37_odd", dict(rows=1030, C=37, off=3)),
    ("c1001_odd", dict(rows=33, C=1001)),
    ("c2048_unaligned", dict(rows=33, C=2048, off=1)),
    ("no_gate", dict(rows=30, C=512, z=False)),
    ("no_post", dict(rows=30, C=512, w1=False)),
    ("no_scale", dict(rows=30, C=512, sc=False)),
    ("no_stream", dict(rows=30, C=512, x=False)),
    ("no_stream_f32", dict(rows=30, C=512, x=False, stream="f32")),
    ("no_pre", dict(rows=30, C=512, w2=False)),
    ("only_add", dict(rows=30, C=512, w1=False, z=False, sc=False, w2=False)),
    ("only_norm", dict(rows=30, C=512, w1=False, z=False, sc=False, x=False)),
    ("only_dn", dict(rows=30, C=512, dr=False)),
    ("only_dr", dict(rows=30, C=512, dn=False)),
    ("wide_bare", dict(rows=3, C=8196, w1=False, z=False, sc=False, x=False)),
    ("stream_f32", dict(rows=70, C=1024, stream="f32")),
    ("stream_f32_odd", dict(rows=70, C=777, stream="f32", off=1)),
    ("stream_f32_wide", dict(rows=4, C=8300, stream="f32")),
    ("sigmoid", dict(rows=30, C=512, act="sigmoid")),
    ("gate_none", dict(rows=30, C=512, act="none")),
    ("f32", dict(rows=70, C=2048, dtype="f32")),
    ("f32_odd", dict(rows=70, C=1001, dtype="f32", off=1)),
    ("f32_wide", dict(rows=3, C=8500, dtype="f32")),
    ("f32_many", dict(rows=3000, C=96, dtype="f32")),
    ("large_values", dict(rows=20, C=512, big=1e4)),
    ("rows_empty", dict(rows=0, C=512)),
]


def _case(name, rows, C, dtype="bf16", stream=None, off=0, act="silu", big=1.0, x=True, z=True,
          w1=True, sc=True, w2=True, dr=True, dn=True):
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    stream = stream or dtype
    c = {"y": rnd(rng, dtype, rows, C, scale=0.5 * big),
         "x": rnd(rng, stream, rows, C, scale=big) if x else None,
         "z": rnd(rng, dtype, rows, C) if z else None,
         "w1": 1 + rnd(rng, "f32", C, scale=0.1) if w1 else None,
         "sc": 0.5 + rnd(rng, "f32", C, scale=0.1) if sc else None,
         "w2": 1 + rnd(rng, "f32", C, scale=0.1) if w2 else None,
         "dr": rnd(rng, stream, rows, C) if dr else None,
         "dn": rnd(rng, dtype, rows, C) if dn and w2 else None}
    c.update(dtype=dtype, stream=stream, off=off, act=act)
    return c


def _inputs(c):
    def put(name, d):
        x = c[name]
        return column_slice(x, dt(d), 1, c["off"], c["off"]) if c["off"] else dev(x, dt(d))

    y, z, x = put("y", c["dtype"]), put("z", c["dtype"]), put("x", c["stream"])
    return (y, x, dev(c["w2"])), dict(post_weight=dev(c["w1"]), z=z, scale=dev(c["sc"]),
                                      activation=c["act"], stream_dtype=dt(c["stream"]))


def _hold(name, got, want, dtype, terms=0.0):
    """The kernels compute in fp32 (1e-5 of the tensor's largest, the repository's bar), and
    round once: half a step of the value for bf16.  Where terms cancel, each carries at most 16
    roundings of 2^-24: 1e-6 of the sum of their absolute values."""
    assert (got is None) == (want is None), name
    if want is None or want.size == 0:
        return
    got = host(got)
    assert np.all(np.isfinite(got)), name
    h = HALF[dtype] if dtype == "bf16" else 0.0
    over = np.abs(got - want) - (h * np.abs(want) * (1 + 1e-5) + 1e-5 * np.max(np.abs(want)) + 1e-6 * terms)
    assert np.max(over) <= 0, (name, np.max(over), np.max(np.abs(got - want)))


@pytest.mark.parametrize("name,kw", CASES, ids=[c[0] for c in CASES])
def test_forward_and_backward(name, kw):
    import paper_2506_02475_amd as comba

    c = _case(name, **kw)
    args, kws = _inputs(c)
    r, n = comba.comba_block_norm_fwd(*args, **kws)
    ops = [c[k] for k in ("y", "x", "z", "w1", "sc", "w2")]
    want_r, want_n = ref.block_fwd(*ops, c["act"])
    assert r.dtype is dt(c["stream"])
    _hold("r", r, want_r, c["stream"])
    _hold("n", n, want_n, c["dtype"])
    got = comba.comba_block_norm_bwd(*args, dev(c["dr"], dt(c["stream"])), dev(c["dn"], dt(c["dtype"])),
                                     **kws)
    want = ref.block_bwd(*ops, c["dr"], c["dn"], c["act"])
    terms = ref.block_bwd(*ops, c["dr"], c["dn"], c["act"], terms=True)
    types = {"dy": c["dtype"], "dz": c["dtype"], "dx": c["stream"]}
    for k, g in got.items():
        _hold(k, g, want.get(k), types.get(k, "f32"), terms.get(k))


def test_two_calls_give_the_same_bits():
    import paper_2506_02475_amd as comba

    c = _case("twice", rows=5000, C=640)
    args, kws = _inputs(c)
    dr, dn = dev(c["dr"], dt("bf16")), dev(c["dn"], dt("bf16"))
    a = comba.comba_block_norm_bwd(*args, dr, dn, **kws)
    b = comba.comba_block_norm_bwd(*args, dr, dn, **kws)
    for k in a:
        assert bool((a[k] == b[k]).all()), k
