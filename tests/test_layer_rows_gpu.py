"""Rows that lie far apart: one token of each of a batch's long rows, as a slice of the
projection leaves it.  The calls give what they give on a contiguous copy, bit for bit
(the same kernels read the same values), also where offsets pass 32 bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


D, N, B = 64, 16, 3


def _far(dtype, stride, width=D, tokens=False):
    """Rows [B, width] ([B, 1, width]) `stride` elements apart in one buffer."""
    import torch

    buf = torch.empty(stride * (B - 1) + width + 8, dtype=dtype, device="cuda")
    t = buf[8:].as_strided((B, 1, width) if tokens else (B, width),
                           (stride, stride, 1) if tokens else (stride, 1))
    t.copy_(torch.randn(t.shape, device="cuda"))
    return t


# 2^22 + 64 is a batch of 4,096 tokens of 1,040 channels; 2^30 + 64: the third row's offset
# passes 2^31 elements
STRIDES = [(1 << 22) + 64, (1 << 30) + 64]


@pytest.mark.parametrize("stride", STRIDES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_convolution_and_norm(dtype, stride):
    import torch

    import paper_2506_02475_amd as comba

    print("far rows: conv, norm", dtype, stride, flush=True)
    torch.manual_seed(1)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, z = _far(dt, stride, tokens=True), _far(dt, stride, tokens=True)
    w, b = torch.randn(D, 4, device="cuda"), torch.randn(D, device="cuda")
    h0, dy = torch.randn(B, 3, D, device="cuda").to(dt), torch.randn(B, 1, D, device="cuda").to(dt)

    def calls(x, z):
        out = list(comba.comba_conv_fwd(x, w, b, h0))
        gr = comba.comba_conv_bwd(x, w, b, h0, dy)
        out += [gr[k] for k in sorted(gr)]
        pool = h0.clone()
        out += [comba.comba_conv_step(x[:, 0], w, b, pool), pool]
        out.append(comba.comba_group_norm_fwd(x, 4, b, b, z))
        gr = comba.comba_group_norm_bwd(x, 4, b, b, z, dy)
        return out + [gr[k] for k in sorted(gr)]

    for i, (got, want) in enumerate(zip(calls(x, z), calls(x.contiguous(), z.contiguous()))):
        assert torch.equal(got, want), i


@pytest.mark.parametrize("stride", STRIDES)
def test_scan_step(stride):
    import torch

    import paper_2506_02475_amd as comba

    print("far rows: scan step", stride, flush=True)
    torch.manual_seed(2)
    bf = torch.bfloat16
    u, delta, z = (_far(bf, stride) for _ in range(3))
    Bm, Cm = _far(bf, stride, N), _far(bf, stride, N)
    A, b = -torch.rand(D, N, device="cuda"), torch.randn(D, device="cuda")
    state = torch.randn(B, D, N, device="cuda")

    def step(*t):
        s = state.clone()
        u, delta, Bm, Cm, z = t
        return comba.comba_select_step(u, delta, A, Bm, Cm, b, z, b, s), s

    ins = (u, delta, Bm, Cm, z)
    for got, want in zip(step(*ins), step(*(t.contiguous() for t in ins))):
        assert torch.equal(got, want)


def test_scan_refuses_far_rows_by_name():
    import torch

    import paper_2506_02475_amd as comba

    z = _far(torch.bfloat16, STRIDES[0], tokens=True)
    u, Bm = z.contiguous(), torch.zeros(B, 1, N, device="cuda", dtype=z.dtype)
    A = -torch.rand(D, N, device="cuda")
    with pytest.raises(comba.CombaError, match="rows of z .* 4194304"):
        comba.comba_select_fwd(u, u, A, Bm, Bm, None, z)
