"""Rows of the selective scan that are cut into segments: that they are cut, and packed
batches in which whole sequences longer than a segment are worked on before the cut one,
against the fp64 reference.

How a call was cut shows in its forward workspace: a state and a sum of steps per channel
and work row, nothing where no sequence is cut."""
import ctypes

import numpy as np
import pytest

import test_layer_ops_gpu as ops

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _work_rows(B=1, T=0, D=0, N=16, G=1, lens=None, **_):
    """Work rows of a forward that is cut, 0 of one that is not; and the backward's cut."""
    import paper_2506_02475_amd as comba

    lib = comba.load_library()
    s = comba.CombaSelectShape(B=B, T=T, D=D, N=N, G=G, num_seqs=B, in_dtype=comba.COMBA_BF16,
                               delta_softplus=1)
    if lens is not None:
        cu = np.cumsum([0] + list(lens)).astype(np.int32)
        s.B, s.T, s.num_seqs = 1, int(cu[-1]), len(lens)
        s.cu_seqlens, s.cu_seqlens_host = 256, cu.ctypes.data  # (the first is not read here)
    S = s.num_seqs
    block = 512 // N
    parts = G * -(-(D // G) // block)

    def up(n):
        return -(-n // 256) * 256

    fwd = lib.comba_select_fwd_workspace_bytes(ctypes.byref(s))
    bwd = lib.comba_select_bwd_workspace_bytes(ctypes.byref(s))
    rows = [r for r in range(2000) if fwd == up(r * D * N * 4) + up(r * D * 4) + 256][0]
    whole = up(parts * s.T * 2 * N * 4) + up(S * D * (N + 2) * 4) + 256
    return rows, bwd > whole


def test_the_cut_cases_are_cut():
    for name, kw in ops.SEGMENTED:
        if name == "packed_mixed":  # fills the CUs: its sequences stay whole
            continue
        rows, bwd = _work_rows(**kw)
        S = len(kw.get("lens") or [0] * kw["B"])
        assert rows > S and bwd, (name, rows, S)


# (name, case, the longest sequence of which is cut and the others not)
WHOLE_FIRST = [
    ("n16", dict(D=3000, N=16, lens=[2000, 600, 150, 30], host=True, dht=True)),
    ("n32", dict(D=1100, N=32, lens=[450, 30, 2000, 0, 100], host=True, dht=True)),
    ("n8_two_whole", dict(D=3000, N=8, lens=[400, 30, 2000, 0, 350], host=True, dht=True,
                          dtype="f32")),
    # more sequences than the host lists
    ("n8_many", dict(D=3000, N=8, lens=[400, 30, 2000, 0, 350] + [3, 0, 9] * 14, host=True)),
]


@pytest.mark.parametrize("name,kw", WHOLE_FIRST, ids=[c[0] for c in WHOLE_FIRST])
def test_whole_sequences_longer_than_a_segment(name, kw):
    print("whole before cut", name, flush=True)
    lens = sorted(kw["lens"])
    rows, bwd = _work_rows(**kw)
    more = rows - len(lens)  # segments beside the first of the one that is cut
    assert bwd and more > 0
    assert (lens[-1] - 1) // more < lens[-2]  # a segment's length, at most: shorter than a whole one
    ops._check_select("whole_first_" + name, kw)
