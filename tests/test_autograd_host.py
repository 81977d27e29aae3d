"""What comba_chunk keeps for its backward and refuses, on the CPU: the training pair stands
in as plain torch functions of the same signatures."""
import numpy as np
import pytest

import paper_2506_02475_amd as comba


@pytest.fixture()
def calls(monkeypatch):
    """o = 2 v, dv = 2 dO, zeros for the rest; the offsets of every call."""
    seen = []

    def fwd(q, k, v, g, beta, d, h0, *, cu_seqlens_host=None, **kw):
        seen.append(np.asarray(cu_seqlens_host).tolist())
        return 2 * v.detach(), v.new_zeros(1), v.new_zeros(7)

    def bwd(q, k, v, g, beta, d, h0, dO, dht, *, cu_seqlens_host=None, **kw):
        seen.append(np.asarray(cu_seqlens_host).tolist())
        zeros = {"d" + n: t.new_zeros(t.shape) for n, t in
                 (("q", q), ("k", k), ("g", g), ("beta", beta), ("d", d))}
        return dict(zeros, dv=2 * dO.detach(), dh0=None)

    monkeypatch.setattr(comba, "comba_chunk_fwd_save", fwd)
    monkeypatch.setattr(comba, "comba_chunk_bwd_saved_in_dtype", bwd)
    return seen


def _args(v):
    import torch

    x, s = torch.zeros(1, 6, 2, 4), torch.zeros(1, 6, 2)
    return x, x, v, s, s, torch.zeros(2)


@pytest.mark.parametrize("tensor", [False, True])
def test_the_backward_has_the_forwards_host_offsets(calls, tensor):
    import torch

    v = torch.randn(1, 6, 2, 4, requires_grad=True)
    cu = torch.tensor([0, 2, 6], dtype=torch.int32)
    host = cu.clone() if tensor else cu.numpy().copy()
    o, _ = comba.comba_chunk(*_args(v), cu_seqlens=cu, cu_seqlens_host=host)
    host[1] = 5  # the caller's buffer, filled for the next batch
    o.sum().backward()
    assert calls == [[0, 2, 6]] * 2
    assert torch.equal(v.grad, torch.full_like(v, 2.0))


def test_second_derivatives_raise(calls):
    """The backward's gradients have no graph of their own: with a product upstream a gradient
    penalty would otherwise lose the operator's part without a word."""
    import torch

    s = torch.randn(4, requires_grad=True)
    v = torch.randn(1, 6, 2, 4) * (s * s)
    o, _ = comba.comba_chunk(*_args(v))
    g, = torch.autograd.grad(o.square().sum(), s, create_graph=True)
    assert torch.isfinite(g).all()
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()
