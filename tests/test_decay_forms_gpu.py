"""Linear attention with a decay per head: head sizes, types and cut sequences that no other test
takes through the kernels, and sums of decays far below what a state holds."""
import math

import numpy as np
import pytest

import test_decay_gpu as decay
from block_helpers import dev, dt, hold

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


FORMS = [
    ("d64_d256", dict(B=1, T=140, H=2, dk=64, dv=256, dht=True)),
    ("d40_d201_odd", dict(B=2, T=77, H=2, dk=40, dv=201, off=3, dht=True)),
    ("d256_d128", dict(B=1, T=140, H=2, dk=256, dv=128, dht=True)),
    ("d200_d100_odd", dict(B=1, T=130, H=2, heads=(1, 2, 1), dk=200, dv=100, off=1, dht=True)),
    ("d129_d64", dict(B=1, T=65, H=1, dk=129, dv=64)),
    ("f32_d128_d64", dict(B=1, T=130, H=2, dk=128, dv=64, dtype="f32", dht=True)),
    ("f32_d100_d40_odd", dict(B=2, T=70, H=2, heads=(2, 1, 2), dk=100, dv=40, dtype="f32", off=1)),
    ("f32_d64_d256", dict(B=1, T=70, H=2, dk=64, dv=256, dtype="f32", dht=True)),
    ("f32_d256_d64", dict(B=1, T=70, H=2, dk=256, dv=64, dtype="f32", dht=True)),
    ("f32_cut_d128", dict(B=1, T=1300, H=1, dk=128, dv=64, dtype="f32", tau=300.0, dht=True)),
    ("f32_cut_d256", dict(H=1, dk=256, dv=40, lens=[3, 900, 650], dtype="f32", tau=300.0, dht=True)),
    ("f32_cut_odd", dict(B=1, T=1001, H=1, dk=65, dv=33, dtype="f32", off=1, tau=300.0)),
    ("cut_shared", dict(B=1, T=1200, H=2, heads=(1, 2, 1), dk=128, dv=64, tau=300.0, dht=True)),
    ("cut_gate_head", dict(B=1, T=1200, H=2, dk=64, dv=64, gate="head", tau=300.0, dht=True)),
]


@pytest.mark.parametrize("name,kw", FORMS, ids=[c[0] for c in FORMS])
def test_forward(name, kw):
    decay.test_forward(name, kw)


@pytest.mark.parametrize("name,kw", FORMS, ids=[c[0] for c in FORMS])
def test_backward(name, kw):
    decay.test_backward(name, kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_resets_and_then_small_decays(dtype):
    """58 of a chunk's first rows reset: its sums of decays reach 58 times 128 log2(e), 10,711, and
    the rows behind them have decays of about 1/20.  Sums below 2^14 are fp32 within 2^-11, a
    difference of two within 2^-10 and a weight within ln(2) 2^-10 of itself: ln(2) / 4 of bf16's
    half step (2^-8), so much more of the terms' absolute values.  (fp32 subtracts sums of two
    floats: its own bound holds as it is.)"""
    import paper_2506_02475_amd as comba

    c = decay._case("many_resets", B=1, T=200, H=3, dk=64, dv=64, gate="f32", dtype=dtype, dht=True)
    g = c["g"]
    for start, n, h in ((0, 58, 0), (64, 58, 0), (128, 60, 0), (0, 30, 1), (96, 32, 1), (66, 61, 2)):
        g[start:start + n, h] = -np.inf
    args = decay._inputs(c)
    o, ht, ws = comba.comba_decay_fwd_save(*args, scale=c["scale"])
    more = 1 + (math.log(2) / 4 if dtype == "bf16" else 0)
    (want, want_t), (mag, _) = decay._fwd(c), decay._fwd(decay._abs(c))
    hold("o", o, want, more * mag, dtype)
    hold("ht", ht, want_t, None, "f32")
    do = dev(c["do"], dt(dtype)).reshape(c["lead"] + c["do"].shape[1:])
    got = comba.comba_decay_bwd(*args, do, dev(c["dht"]), workspace=ws, scale=c["scale"])
    want, mag = decay._bwd(c), decay._bwd(decay._abs(c))
    for n in ("dq", "dk", "dv"):
        hold(n, got[n], want[n], more * mag[n], dtype)
    hold("dg", got["dg"], want["dg"], more * mag["dg"], dtype, inner=2)
    hold("dh0", got["dh0"], want["dh0"], None, "f32")
