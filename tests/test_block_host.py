"""Host-side checks of include/comba_block.h: every declared symbol is exported and bound, bad
arguments are refused before any launch, and what the differentiable calls keep and refuse
(no GPU needed)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2506_02475_amd as comba
from paper_2506_02475_amd import block

pytestmark = pytest.mark.skipif(not os.path.exists(comba.library_path()),
                                reason="libcomba.so not built")

ENULL, ESHAPE, EDTYPE, EALIGN, EWS = 1, 2, 3, 4, 5
FAKE = 0x100000  # aligned, never dereferenced
BIG = 1 << 45
BF16, F32 = comba.COMBA_BF16, comba.COMBA_F32


def _struct(cls, **over):
    host = over.pop("host", None)
    s = cls(**over)
    if host is not None:
        a = np.asarray(host, np.int32)
        s.cu_seqlens_host = a.ctypes.data
        s._keep = a
    return s


def decay(**over):
    base = dict(B=2, T=10, H=4, Hq=4, Hk=2, Hv=1, dk=16, dv=24, num_seqs=2, in_dtype=BF16,
                g_dtype=BF16, scale=1.0)
    return _struct(comba.CombaDecayShape, **dict(base, **over))


def norm(**over):
    base = dict(rows=5, C=64, dtype=BF16, x_dtype=F32, activation=1, eps=1e-6)
    return _struct(comba.CombaBlockNormShape, **dict(base, **over))


CALLS = {
    "comba_decay_fwd": ("q k v g h0? o ht? ws", "ws"),
    "comba_decay_fwd_save": ("q k v g h0? o ht? ws", "ws"),
    "comba_decay_bwd": ("q k v g h0? dO dht? dq dk dv dg? dh0? saved saved_bytes ws", "ws"),
    "comba_decay_step": ("q k v g state slots? num_slots o", None),
    "comba_block_norm_fwd": ("y x? z? w1? s? w2? r n", None),
    "comba_block_norm_bwd": ("y x? z? w1? s? w2? dr? dn? dy dx? dz dw1? ds? dw2? ws", "ws"),
}
SIZES = {"num_slots": 4, "saved_bytes": BIG}


def call(name, shp, ws_bytes=BIG, **over):
    names, ws = CALLS[name]
    args = [over.get(n.rstrip("?"), SIZES.get(n, FAKE)) for n in names.split()]
    if ws:
        args.append(ws_bytes)
    return getattr(comba.load_library(), name)(None if shp is None else ctypes.byref(shp), *args,
                                               None)


def shape_of(name, **over):
    if "norm" in name:
        return norm(**over)
    return decay(**(dict(over, T=1) if "step" in name and "T" not in over else over))


def test_header_is_exported_and_bound():
    declared = comba.exported_symbols("comba_block.h")
    assert declared == sorted(list(CALLS) + [
        "comba_decay_fwd_workspace_bytes", "comba_decay_save_bytes",
        "comba_decay_bwd_workspace_bytes", "comba_block_norm_workspace_bytes"])
    out = subprocess.run(["nm", "-D", "--defined-only", comba.library_path()],
                         capture_output=True, text=True, check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if line.strip()}
    for name in declared:
        assert name in exported, name
        assert getattr(comba.load_library(), name).argtypes is not None, name
    for name in ("comba_decay", "comba_decay_step", "comba_block_norm"):
        assert name in comba.__all__ and callable(getattr(comba, name))


@pytest.mark.parametrize("name", list(CALLS))
def test_required_pointers(name):
    assert call(name, None) == ENULL
    for n in CALLS[name][0].split():
        if not n.endswith("?") and n not in SIZES:
            assert call(name, shape_of(name), **{n: None}) == ENULL, n


@pytest.mark.parametrize("name", list(CALLS))
def test_misaligned_pointers(name):
    for n in CALLS[name][0].split():
        n = n.rstrip("?")
        if n not in SIZES:
            bad = FAKE + (128 if n in ("ws", "saved") else 1)
            assert call(name, shape_of(name), **{n: bad}) == EALIGN, n


@pytest.mark.parametrize("over,code", [
    (dict(H=0), ESHAPE), (dict(H=65536, Hq=1, Hk=1), ESHAPE), (dict(Hq=3), ESHAPE),
    (dict(Hk=0), ESHAPE), (dict(Hv=8), ESHAPE), (dict(dk=0), ESHAPE), (dict(dk=257), ESHAPE),
    (dict(dv=257), ESHAPE), (dict(dv=-1), ESHAPE), (dict(B=-1), ESHAPE), (dict(num_seqs=3), ESHAPE),
    (dict(in_dtype=7), EDTYPE), (dict(g_dtype=2), EDTYPE), (dict(in_dtype=F32), EDTYPE),
    (dict(g_per_head=1), EDTYPE), (dict(q_row=63), ESHAPE), (dict(k_row=-32), ESHAPE),
    (dict(v_row=23), ESHAPE), (dict(g_row=3), ESHAPE), (dict(q_row=(1 << 22) + 1), ESHAPE),
    (dict(cu_seqlens=FAKE), ESHAPE), (dict(host=[0, 10]), ESHAPE)])
def test_decay_shapes(over, code):
    for name in ("comba_decay_fwd", "comba_decay_fwd_save", "comba_decay_bwd"):
        assert call(name, decay(**over)) == code
    lib = comba.load_library()
    for size in (lib.comba_decay_fwd_workspace_bytes, lib.comba_decay_save_bytes,
                 lib.comba_decay_bwd_workspace_bytes):
        assert size(ctypes.byref(decay(**over))) == 0


@pytest.mark.parametrize("over,code", [
    (dict(C=0), ESHAPE), (dict(rows=-1), ESHAPE), (dict(eps=-1.0), ESHAPE),
    (dict(eps=float("nan")), ESHAPE), (dict(activation=3), ESHAPE), (dict(x_dtype=5), EDTYPE),
    (dict(dtype=F32, x_dtype=BF16), EDTYPE), (dict(y_row=63), ESHAPE), (dict(z_row=-64), ESHAPE),
    (dict(x_row=1), ESHAPE)])
def test_norm_shapes(over, code):
    for name in ("comba_block_norm_fwd", "comba_block_norm_bwd"):
        assert call(name, norm(**over)) == code
    assert comba.load_library().comba_block_norm_workspace_bytes(ctypes.byref(norm(**over))) == 0


def test_constants_of_the_heads_have_no_gradient():
    assert call("comba_decay_bwd", decay(g_per_head=1, g_dtype=F32)) == ESHAPE
    assert call("comba_decay_bwd", decay(g_per_head=1, g_dtype=F32), dg=None, dq=None) == ENULL


@pytest.mark.parametrize("host,ok", [([0, 4, 10], True), ([0, 4, 9], False), ([1, 4, 10], False),
                                     ([0, 11, 10], False)])
def test_host_offsets(host, ok):
    """A well-formed table goes on to the next check (a missing output)."""
    assert call("comba_decay_fwd", decay(B=1, cu_seqlens=FAKE, host=host), o=None) \
        == (ENULL if ok else ESHAPE)


def test_steps_take_one_token_and_no_offsets():
    name = "comba_decay_step"
    assert call(name, decay(T=2)) == ESHAPE
    assert call(name, decay(B=1, T=1, cu_seqlens=FAKE, num_seqs=1)) == ESHAPE
    assert call(name, decay(T=1), num_slots=-1) == ESHAPE
    for r in ("q_row", "k_row", "v_row", "g_row"):  # rows of a step lie any distance apart
        assert call(name, decay(T=1, **{r: 1 << 23}), o=None) == ENULL
        assert call(name, decay(T=1, **{r: 1 << 60}), o=None) == ESHAPE


def test_a_step_takes_fewer_than_2_24_rows():
    """A launch holds fewer than 2^32 threads along a dimension, a step 256 a row."""
    one = dict(T=1, H=1, Hq=1, Hk=1, Hv=1, dk=1, dv=1)
    for n, code in (((1 << 24) - 1, ENULL), (1 << 24, ESHAPE)):
        assert call("comba_decay_step", decay(B=n, num_seqs=n, **one), o=None) == code


def test_workspaces():
    lib = comba.load_library()
    for name, size, shp in (
            ("comba_decay_fwd", lib.comba_decay_fwd_workspace_bytes, decay()),
            ("comba_decay_fwd_save", lib.comba_decay_save_bytes, decay()),
            ("comba_decay_bwd", lib.comba_decay_bwd_workspace_bytes, decay()),
            ("comba_block_norm_bwd", lib.comba_block_norm_workspace_bytes, norm())):
        n = size(ctypes.byref(shp))
        assert n > 0
        assert call(name, shp, ws_bytes=n - 1) == EWS, name
    # the states kept for the backward: one per 64 tokens and sequence, in blocks of 16 x 16
    shp = decay()
    kept = 2 * 1 * 4 * 16 * 32 * 2
    assert lib.comba_decay_save_bytes(ctypes.byref(shp)) >= kept
    assert call("comba_decay_bwd", shp, saved_bytes=kept - 1) == EWS
    # shared heads: fp32 gradients of every state head's q, k, v
    whole = lib.comba_decay_bwd_workspace_bytes(ctypes.byref(decay(Hk=4, Hv=4)))
    some = lib.comba_decay_bwd_workspace_bytes(ctypes.byref(decay()))
    assert some >= whole + 20 * 4 * (16 + 24) * 4


def test_large_calls_are_refused_by_shape():
    """A launch holds fewer than 2^31 threads, and a chunk's rows fewer than 2^31 bytes: more is
    refused before the first of a call's launches."""
    most = (1 << 31) // 512 - 64
    for name in ("comba_decay_fwd", "comba_decay_bwd"):
        S = 1 << 23
        assert call(name, decay(B=S, num_seqs=S, T=1, H=1, Hq=1, Hk=1, Hv=1)) == ESHAPE
        assert call(name, decay(B=1, num_seqs=1, T=1, H=32768, Hq=1, Hk=1, dv=256)) == ESHAPE
        fits = decay(B=1, num_seqs=1, T=64 * (most // 64), H=16, Hq=1, Hk=1, dv=32)
        assert call(name, fits, q=None) == ENULL


def test_tokens_need_a_sequence():
    assert call("comba_decay_fwd", decay(B=1, num_seqs=0, cu_seqlens=FAKE)) == ESHAPE


def test_binding_refuses_before_the_library():
    import torch

    x, g = torch.zeros(2, 3, 4, 8), torch.zeros(2, 3, 4)
    with pytest.raises(comba.CombaError, match="GPU"):
        comba.comba_decay_fwd(x, x, x, g)
    with pytest.raises(comba.CombaError, match="GPU"):
        comba.comba_decay_step(x[:, 0], x[:, 0], x[:, 0], g[:, 0], torch.zeros(2, 4, 8, 8))
    with pytest.raises(comba.CombaError, match="GPU"):
        comba.comba_block_norm_fwd(torch.zeros(3, 8), None, torch.zeros(8))
    with pytest.raises(comba.CombaError, match="q must be"):
        comba.comba_decay_step(x, x, x, g, torch.zeros(2, 4, 8, 8))
    # heads as slices of a wider row
    wide, f = torch.zeros(2, 3, 40), torch.float32
    heads = wide[..., 4:36].unflatten(-1, (4, 8))
    assert block._heads("q", heads, 2, heads.shape[:2], f, -1, 1 << 22) == (4, 8, 40)
    assert block._heads("q", x, 2, x.shape[:2], f, -1, 1 << 22) == (4, 8, 0)
    assert block._heads("q", wide[:, 0, 4:36].unflatten(-1, (4, 8)), 1, (2,), f, -1, None) \
        == (4, 8, 120)
    for bad in (x.transpose(1, 2), heads[:, ::2], heads[..., ::2], heads[:, :, ::2]):
        with pytest.raises(comba.CombaError, match="q"):
            block._heads("q", bad, 2, bad.shape[:2], f, -1, 1 << 22)
    for bad in (x[:, 0].transpose(0, 1), heads[:, 0, :, ::2], x[:1, 0].expand(2, 4, 8)):
        with pytest.raises(comba.CombaError, match="q"):
            block._heads("q", bad, 1, bad.shape[:1], f, -1, None)
    with pytest.raises(comba.CombaError, match="q must be"):
        block._heads("q", x, 2, (2, 4), f, -1, None)
    with pytest.raises(comba.CombaError, match="q must be"):
        block._heads("q", x, 2, (2, 3), torch.bfloat16, -1, None)


class Fakes:
    """The library's calls as plain torch functions: o = 2 v, r = 2 y, n = 3 y; gradients twice
    and three times the outputs'."""

    def __init__(self, monkeypatch):
        self.calls = []
        for name in ("comba_decay_fwd", "comba_decay_fwd_save", "comba_decay_bwd",
                     "comba_block_norm_fwd", "comba_block_norm_bwd"):
            monkeypatch.setattr(block, name, getattr(self, name))

    def _note(self, name, kw):
        host, cu = kw.get("cu_seqlens_host"), kw.get("cu_seqlens")
        self.calls.append((name, None if cu is None else cu.tolist(),
                           None if host is None else np.asarray(host).tolist()))

    def comba_decay_fwd(self, q, k, v, g, h0, **kw):
        self._note("fwd", kw)
        return 2 * v.detach(), v.new_zeros(1, 2, 4, 4)

    def comba_decay_fwd_save(self, q, k, v, g, h0, **kw):
        self._note("fwd_save", kw)
        return 2 * v.detach(), v.new_zeros(1, 2, 4, 4), v.new_zeros(7)

    def comba_decay_bwd(self, q, k, v, g, h0, do, dht=None, *, workspace, need_dg=True,
                        need_dh0=True, **kw):
        self._note("bwd", kw)
        assert workspace.numel() == 7
        return {"dq": q.new_zeros(q.shape), "dk": k.new_zeros(k.shape), "dv": 2 * do.detach(),
                "dg": g.new_zeros(g.shape) if need_dg else None, "dh0": None}

    def comba_block_norm_fwd(self, y, x=None, weight=None, **kw):
        return 2 * y.detach(), None if weight is None else 3 * y.detach()

    def comba_block_norm_bwd(self, y, x, weight, dr, dn, **kw):
        dy = (0 if dr is None else 2 * dr.detach()) + (0 if dn is None else 3 * dn.detach())
        return {"dy": dy, "dx": dr, "dz": None, "dpost_weight": None, "dscale": None,
                "dweight": weight.new_zeros(weight.shape)}


@pytest.fixture()
def fakes(monkeypatch):
    return Fakes(monkeypatch)


def _decay(v, g=None, **packed):
    import torch

    x = torch.zeros(1, v.shape[1], 2, 4)
    return comba.comba_decay(x, x, v, torch.zeros(1, v.shape[1], 2) if g is None else g, **packed)[0]


def test_offsets_written_before_the_backward_raise(fakes):
    import torch

    v = torch.randn(1, 6, 2, 4, requires_grad=True)
    cu = torch.tensor([0, 2, 6], dtype=torch.int32)
    o = _decay(v, cu_seqlens=cu)
    cu.copy_(torch.tensor([0, 5, 6], dtype=torch.int32))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()
    assert [c[0] for c in fakes.calls] == ["fwd_save"]


def test_the_backward_has_the_forwards_host_offsets(fakes):
    import torch

    v = torch.randn(1, 6, 2, 4, requires_grad=True)
    cu = torch.tensor([0, 2, 6], dtype=torch.int32)
    host = cu.numpy().copy()
    o = _decay(v, cu_seqlens=cu, cu_seqlens_host=host)
    host[1] = 5
    o.sum().backward()
    assert [c[1:] for c in fakes.calls] == [([0, 2, 6], [0, 2, 6])] * 2
    assert torch.equal(v.grad, torch.full_like(v, 2.0))


def test_states_are_kept_only_for_a_backward(fakes):
    import torch

    v = torch.randn(1, 6, 2, 4)
    assert not _decay(v).requires_grad
    with torch.no_grad():
        _decay(v.clone().requires_grad_())
    _decay(v.clone().requires_grad_())
    assert [c[0] for c in fakes.calls] == ["fwd", "fwd", "fwd_save"]


def test_trained_constants_of_the_heads_raise(fakes):
    import torch

    v = torch.randn(1, 6, 2, 4, requires_grad=True)
    _decay(v, torch.zeros(2))
    with pytest.raises(comba.CombaError, match="constants"):
        _decay(v, torch.zeros(2, requires_grad=True))


def test_trained_constants_of_the_heads_run_where_no_gradient_is_wanted(fakes):
    """A model may keep them as a parameter: a call without gradients asks for none of theirs."""
    import torch

    v, g = torch.randn(1, 6, 2, 4, requires_grad=True), torch.zeros(2, requires_grad=True)
    with torch.no_grad():
        assert torch.equal(_decay(v, g), 2 * v)
    with torch.inference_mode():
        assert torch.equal(_decay(v, g), 2 * v)
    assert [c[0] for c in fakes.calls] == ["fwd", "fwd"]


@pytest.mark.parametrize("op", ["decay", "norm"])
def test_second_derivatives_and_forward_mode_raise(fakes, op):
    import torch
    import torch.autograd.forward_ad as fwad

    def f(x):
        return _decay(x) if op == "decay" else comba.comba_block_norm(x, None, torch.ones(4))[1]

    u = torch.randn(4, requires_grad=True)
    x = torch.randn(1, 6, 2, 4)
    g, = torch.autograd.grad(f(x * (u * u)).square().sum(), u, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()
    with fwad.dual_level(), torch.no_grad():
        with pytest.raises(RuntimeError, match="forward mode AD|jvp"):
            f(fwad.make_dual(x, torch.ones_like(x)))


def test_norm_gradients_of_either_output(fakes):
    import torch

    y = torch.randn(3, 4, requires_grad=True)
    w = torch.ones(4, requires_grad=True)
    for pick, want in ((lambda r, n: r, 2.0), (lambda r, n: n, 3.0), (lambda r, n: r + n, 5.0)):
        y.grad = None
        pick(*comba.comba_block_norm(y, None, w)).sum().backward()
        assert torch.equal(y.grad, torch.full_like(y, want))
    r, n = comba.comba_block_norm(y, None, None)
    assert n is None and r.requires_grad
