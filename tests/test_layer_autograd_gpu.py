"""The layer's differentiable calls on the GPU where a program reuses its buffers."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _scan_inputs(T, D, N=16, seed=3):
    import torch

    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    bf = torch.bfloat16
    return [rnd(1, T, D).to(bf), rnd(1, T, D).to(bf), -rnd(D, N).exp(), rnd(1, T, N).to(bf),
            rnd(1, T, N).to(bf), rnd(D), rnd(1, T, D).to(bf), rnd(D)]


def test_a_host_buffer_filled_anew_does_not_reach_the_backward():
    """One sequence long enough to be cut: the host offsets choose the backward's work rows."""
    import torch

    import paper_2506_02475_amd as comba

    print("host offsets reused", flush=True)
    ins = [t.requires_grad_() for t in _scan_inputs(1600, 40)]
    w = torch.randn(40, 4, device="cuda", requires_grad=True)
    host = np.array([0, 1500, 1600], np.int32)
    cu = torch.from_numpy(host.copy()).cuda()

    def grads(reuse):
        host[1] = 1500
        y, _ = comba.comba_select(*ins, cu_seqlens=cu, cu_seqlens_host=host)
        v, _ = comba.comba_conv(ins[0], w, cu_seqlens=cu, cu_seqlens_host=host)
        if reuse:
            host[1] = 3
        return torch.autograd.grad((y.float().square().sum(), v.float().square().sum()),
                                   ins + [w])

    for i, (a, b) in enumerate(zip(grads(True), grads(False))):
        assert torch.equal(a, b), i


def test_device_offsets_filled_anew_are_refused():
    import torch

    import paper_2506_02475_amd as comba

    print("device offsets reused", flush=True)
    ins = [t.requires_grad_() for t in _scan_inputs(90, 24)]
    w = torch.randn(24, 4, device="cuda")
    for call in (lambda c: comba.comba_select(*ins, cu_seqlens=c)[0],
                 lambda c: comba.comba_conv(ins[0], w, cu_seqlens=c)[0]):
        cu = torch.tensor([0, 30, 90], dtype=torch.int32, device="cuda")
        y = call(cu)
        cu[1] = 60
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.float().sum().backward()
