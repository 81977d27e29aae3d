"""Norms that a call does not have (no weight, no post weight, no gradient of n) take no part in
its gradients: infinities in what they would have divided reach nothing."""
import numpy as np
import pytest

from block_helpers import dev, dt, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# a team of 16 lanes, a wave, workgroups, rows as loaded, rows from the caches; aligned and odd
WIDTHS = [64, 37, 500, 2048, 4096, 5000, 7001, 8200, 8203]


def _case(C, dtype, stream, rows=5):
    """Inputs, and the same with an infinity in x and another in y, in rows of their own."""
    rng = np.random.default_rng(C)
    t = {n: rnd(rng, dtype, rows, C) for n in ("y", "z", "dn")}
    t.update({n: rnd(rng, stream, rows, C) for n in ("x", "dr")})
    p = {n: dev(1 + rnd(rng, "f32", C, scale=0.1)) for n in ("w1", "sc", "w2")}
    x, y = t["x"].copy(), t["y"].copy()
    x[1, C // 2], y[3, C // 3] = np.inf, -np.inf
    types = {"x": stream, "dr": stream}
    t = {n: dev(v, dt(types.get(n, dtype))) for n, v in t.items()}
    return t, p, dev(x, dt(stream)), dev(y, dt(dtype))


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_without_weight_the_gradients_do_not_read_x(C, dtype, stream):
    import torch

    import paper_2506_02475_amd as comba

    t, p, x, _ = _case(C, dtype, stream)
    kw = dict(post_weight=p["w1"], z=t["z"], scale=p["sc"])
    got = comba.comba_block_norm_bwd(t["y"], x, None, t["dr"], None, **kw)
    want = comba.comba_block_norm_bwd(t["y"], t["x"], None, t["dr"], None, **kw)
    assert torch.equal(got["dx"], t["dr"])
    for n in ("dy", "dz", "dpost_weight", "dscale"):
        assert torch.equal(got[n], want[n]) and torch.isfinite(got[n]).all(), n


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("f32", "f32")])
def test_without_a_gradient_of_n_its_norm_takes_no_part(C, dtype, stream):
    import torch

    import paper_2506_02475_amd as comba

    t, p, x, _ = _case(C, dtype, stream)
    kw = dict(post_weight=p["w1"], z=t["z"], scale=p["sc"])
    got = comba.comba_block_norm_bwd(t["y"], x, p["w2"], t["dr"], None, **kw)
    want = comba.comba_block_norm_bwd(t["y"], t["x"], None, t["dr"], None, **kw)
    assert not got.pop("dweight").any()
    for n in ("dx", "dy", "dz", "dpost_weight", "dscale"):
        assert torch.equal(got[n], want[n]), n
