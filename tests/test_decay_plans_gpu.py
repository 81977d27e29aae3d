"""Linear attention with a decay per head: whole sequences and the same ones cut into segments,
and either's kept states for the other's backward."""
import pytest

import test_decay_gpu as decay
from block_helpers import dev, dt, hold, packed

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# whole with host offsets, as if of one sequence without them (and then cut)
LENS = [500, 0, 400, 300]


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 64, 64), ("bf16", 128, 48), ("f32", 64, 64)])
@pytest.mark.parametrize("saved,then", [(False, True), (True, False)], ids=["cut_whole", "whole_cut"])
def test_whole_and_cut(dtype, dk, dv, saved, then):
    """``saved``, ``then``: whether the forward and the backward know the offsets on the host; the
    states kept by either plan serve both."""
    import paper_2506_02475_amd as comba

    c = decay._case("plans", H=1, dk=dk, dv=dv, lens=LENS, dht=True, tau=300.0, dtype=dtype)
    args, kw = decay._inputs(c), [dict(scale=0.7, **packed(LENS, h)) for h in (False, True)]
    o, ht, ws = comba.comba_decay_fwd_save(*args, **kw[saved])
    other = comba.comba_decay_fwd_save(*args, **kw[not saved])[2]
    assert (ws.numel() > other.numel()) == then  # a plan with segments holds their ends
    want, want_t = decay._fwd(c)
    mag, _ = decay._fwd(decay._abs(c))
    hold("o", o, want, mag, dtype)
    hold("ht", ht, want_t, None, "f32")
    do = dev(c["do"], dt(dtype)).reshape(c["lead"] + c["do"].shape[1:])
    got = comba.comba_decay_bwd(*args, do, dev(c["dht"]), workspace=ws, **kw[then])
    want, mag = decay._bwd(c), decay._bwd(decay._abs(c))
    for n in ("dq", "dk", "dv"):
        hold(n, got[n], want[n], mag[n], dtype)
    hold("dg", got["dg"], want["dg"], mag["dg"], dtype, inner=2)
    hold("dh0", got["dh0"], want["dh0"], None, "f32")


def test_a_workspace_without_the_states_is_refused():
    import torch

    import paper_2506_02475_amd as comba

    c = decay._case("small", H=1, dk=64, dv=64, lens=LENS)
    args, kw = decay._inputs(c), packed(LENS, True)
    do = torch.zeros(1, sum(LENS), 1, 64, device="cuda", dtype=torch.bfloat16)
    ws = comba.comba_decay_fwd_save(*args, **kw)[2]
    kept = (sum(LENS) // 64 + len(LENS)) * (64 * 64 * 2 + 16 * 4)  # fp16 and a scale a block
    for bad in (None, ws[:kept - 1]):
        with pytest.raises(comba.CombaError, match="workspace"):
            comba.comba_decay_bwd(*args, do, workspace=bad, **kw)
    comba.comba_decay_bwd(*args, do, workspace=ws[:kept], **kw)
