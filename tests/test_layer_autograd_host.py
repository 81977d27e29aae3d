"""What the layer's differentiable calls keep and refuse, on the CPU: the library's calls
stand in as plain torch functions of the same signatures, so that only the autograd
functions themselves are run."""
import numpy as np
import pytest

import paper_2506_02475_amd as comba
from paper_2506_02475_amd import layer


class Fakes:
    """Forwards y = 2 x with states of zeros; backwards dx = 2 dy, zeros for the rest.
    ``calls``: the name and offsets of every call."""

    def __init__(self, monkeypatch):
        self.calls = []
        for name in ("comba_conv_fwd", "comba_conv_bwd", "comba_select_fwd",
                     "comba_select_fwd_save", "comba_select_bwd", "comba_group_norm_fwd",
                     "comba_group_norm_bwd"):
            monkeypatch.setattr(layer, name, getattr(self, name))

    def _note(self, name, kw):
        host = kw.get("cu_seqlens_host")
        cu = kw.get("cu_seqlens")
        self.calls.append((name, None if cu is None else cu.tolist(),
                           None if host is None else np.asarray(host).tolist()))

    def comba_conv_fwd(self, x, w, bias, h0, **kw):
        self._note("conv_fwd", kw)
        return 2 * x.detach(), x.new_zeros(1, 3, x.shape[-1])

    def comba_conv_bwd(self, x, w, bias, h0, dy, dht=None, *, need_dh0=True, **kw):
        self._note("conv_bwd", kw)
        return {"dx": 2 * dy.detach(), "dw": w.new_zeros(w.shape), "dbias": None, "dh0": None}

    def _select(self, name, u, A, kw):
        self._note(name, kw)
        return 2 * u.detach(), u.new_zeros(1, u.shape[-1], A.shape[1]), u.new_zeros(7)

    def comba_select_fwd(self, u, delta, A, *rest, **kw):
        return self._select("select_fwd", u, A, kw)[:2]

    def comba_select_fwd_save(self, u, delta, A, *rest, **kw):
        return self._select("select_fwd_save", u, A, kw)

    def comba_select_bwd(self, u, delta, A, B, C, D, z, bias, h0, dy, dht=None, *, workspace,
                         need_dh0=True, **kw):
        self._note("select_bwd", kw)
        assert workspace.numel() == 7
        z = {"d" + n: t.new_zeros(t.shape) for n, t in (("delta", delta), ("A", A), ("B", B),
                                                        ("C", C))}
        return dict(z, du=2 * dy.detach(), dD=None, dz=None, ddelta_bias=None, dh0=None)

    def comba_group_norm_fwd(self, x, groups, weight, bias, z, **kw):
        self._note("norm_fwd", kw)
        return 2 * x.detach()

    def comba_group_norm_bwd(self, x, groups, weight, bias, z, dy, **kw):
        self._note("norm_bwd", kw)
        return {"dx": 2 * dy.detach(), "dweight": None, "dbias": None, "dz": None}


@pytest.fixture()
def fakes(monkeypatch):
    return Fakes(monkeypatch)


def _ops(x, **packed):
    """(name, output) of each differentiable call on x [1,T,8]."""
    import torch

    w, A, b = torch.zeros(8, 4), torch.zeros(8, 16), torch.zeros(x.shape[:2] + (16,))
    ops = {"conv": lambda: comba.comba_conv(x, w, **packed)[0],
           "select": lambda: comba.comba_select(x, x, A, b, b, **packed)[0]}
    if not packed:
        ops["norm"] = lambda: comba.comba_group_norm(x, 2)
    return ops


@pytest.mark.parametrize("op", ["conv", "select"])
def test_offsets_written_before_the_backward_raise(fakes, op):
    import torch

    x = torch.randn(1, 6, 8, requires_grad=True)
    cu = torch.tensor([0, 2, 6], dtype=torch.int32)
    y = _ops(x, cu_seqlens=cu)[op]()
    cu.copy_(torch.tensor([0, 5, 6], dtype=torch.int32))  # the next batch's
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    assert not any("bwd" in c[0] for c in fakes.calls)


@pytest.mark.parametrize("tensor", [False, True])
@pytest.mark.parametrize("op", ["conv", "select"])
def test_the_backward_has_the_forwards_host_offsets(fakes, op, tensor):
    import torch

    x = torch.randn(1, 6, 8, requires_grad=True)
    cu = torch.tensor([0, 2, 6], dtype=torch.int32)
    host = cu.clone() if tensor else cu.numpy().copy()
    y = _ops(x, cu_seqlens=cu, cu_seqlens_host=host)[op]()
    host[1] = 5  # the caller's buffer, filled for the next batch
    y.sum().backward()
    assert [c[1:] for c in fakes.calls] == [([0, 2, 6], [0, 2, 6])] * 2
    assert torch.equal(x.grad, torch.full_like(x, 2.0))


@pytest.mark.parametrize("op", ["conv", "select", "norm"])
def test_second_derivatives_raise(fakes, op):
    """The backward's gradients have no graph of their own: with a product upstream a gradient
    penalty would otherwise lose the operator's part without a word."""
    import torch

    v = torch.randn(8, requires_grad=True)
    x = torch.randn(1, 6, 8)
    y = _ops(x * (v * v))[op]()
    g, = torch.autograd.grad(y.square().sum(), v, create_graph=True)
    assert torch.isfinite(g).all()
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()


@pytest.mark.parametrize("op", ["conv", "select", "norm"])
def test_forward_mode_raises_without_grad_mode_too(fakes, op):
    """Forward-mode differentiation does not depend on grad mode: a result without its tangent
    would read as a derivative of zero."""
    import torch
    import torch.autograd.forward_ad as fwad

    with fwad.dual_level(), torch.no_grad():
        x = fwad.make_dual(torch.randn(1, 6, 8), torch.ones(1, 6, 8))
        with pytest.raises(RuntimeError, match="forward mode AD|jvp"):
            _ops(x)[op]()


def test_states_are_kept_only_for_a_backward(fakes):
    import torch

    def names(x):
        del fakes.calls[:]
        _ops(x)["select"]()
        return [c[0] for c in fakes.calls]

    x = torch.randn(1, 6, 8)
    assert names(x) == ["select_fwd"]  # grad mode, but nothing to differentiate
    assert names(x.clone().requires_grad_()) == ["select_fwd_save"]
    with torch.no_grad():
        assert names(x.clone().requires_grad_()) == ["select_fwd"]
    with torch.inference_mode():
        assert names(x) == ["select_fwd"]
    y = _ops(x)["select"]()
    assert not y.requires_grad
