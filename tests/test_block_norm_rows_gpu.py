"""Norms after and before a block: rows enough that every kind of team (16 lanes, a wave,
workgroups) walks more than one, the last walk not full, and widths between the powers of two."""
import pytest

import test_block_norm_gpu as norm

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# teams: 16,384 or 8,192 of 16 lanes, 4,096 or 2,048 of a wave, 1,024 or 512 of four, 256 wider
CASES = [
    ("lanes16", dict(rows=16390, C=64)),
    ("lanes16_odd", dict(rows=16387, C=37, off=3)),
    ("lanes16_two", dict(rows=8195, C=96)),
    ("lanes16_two_f32", dict(rows=8193, C=127, dtype="f32")),
    ("wave", dict(rows=4100, C=256)),
    ("wave_odd", dict(rows=4099, C=201, off=1, stream="f32")),
    ("wave_two", dict(rows=2051, C=500)),
    ("wave_two_odd", dict(rows=2050, C=511)),
    ("waves4", dict(rows=1030, C=1000, off=4)),
    ("waves4_f32", dict(rows=2051, C=1024, dtype="f32")),
    ("waves4_odd", dict(rows=1027, C=601, off=1)),
    ("waves4_two", dict(rows=515, C=2048)),
    ("waves4_two_unaligned", dict(rows=515, C=2048, off=1, stream="f32")),
    ("waves8", dict(rows=259, C=2560)),
    ("waves8_odd", dict(rows=515, C=4095)),
    ("c5120", dict(rows=259, C=5120)),
    ("c5120_f32", dict(rows=259, C=5120, dtype="f32")),
    ("c6144_stream_f32", dict(rows=259, C=6144, stream="f32")),
    ("c7168", dict(rows=515, C=7168)),
    ("c5001_odd", dict(rows=259, C=5001)),
    ("c7001_odd_f32", dict(rows=259, C=7001, dtype="f32")),
    ("c8191_stream_f32", dict(rows=5, C=8191, stream="f32", off=1)),
    ("c8192_unaligned", dict(rows=259, C=8192, off=1)),
    ("c4097_bare", dict(rows=3, C=4097, w1=False, z=False, sc=False, x=False)),
    ("c6144_add_norm", dict(rows=259, C=6144, w1=False, z=False, sc=False, stream="f32")),
    ("c6000_no_pre", dict(rows=259, C=6000, w2=False)),
    ("c12288", dict(rows=259, C=12288)),
    ("c16385_odd_f32", dict(rows=3, C=16385, dtype="f32")),
]


@pytest.mark.parametrize("name,kw", CASES, ids=[c[0] for c in CASES])
def test_forward_and_backward(name, kw):
    norm.test_forward_and_backward(name, kw)
