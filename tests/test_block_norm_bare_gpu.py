"""Without a norm after the block, the gradient of its output reads that output in no other way than
through the norm before the next block."""
import pytest

from test_block_norm_absent_gpu import WIDTHS, _case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_without_post_weight_dy_does_not_read_y(C, dtype, stream):
    """An infinity in y: dy and dx are those of the finite y, bit for bit; dz and dscale, which
    multiply y, are infinite in its own place alone."""
    import torch

    import paper_2506_02475_amd as comba

    t, p, _, y = _case(C, dtype, stream)
    at = torch.isinf(y)
    for z in (t["z"], None):
        kw = dict(z=z, scale=p["sc"])
        got = comba.comba_block_norm_bwd(y, t["x"], None, t["dr"], None, **kw)
        want = comba.comba_block_norm_bwd(t["y"], t["x"], None, t["dr"], None, **kw)
        for n in ("dy", "dx"):
            assert torch.equal(got[n], want[n]) and torch.isfinite(got[n]).all(), n
        assert torch.equal(got["dscale"][~at.any(0)], want["dscale"][~at.any(0)])
        if z is not None:
            assert torch.equal(got["dz"][~at], want["dz"][~at])
