"""Host-side checks of include/comba_layer.h: every declared symbol is exported and
bound, and bad arguments are refused before any launch (no GPU needed)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2506_02475_amd as comba

pytestmark = pytest.mark.skipif(not os.path.exists(comba.library_path()),
                                reason="libcomba.so not built")

OK, ENULL, ESHAPE, EDTYPE, EALIGN, EWS = 0, 1, 2, 3, 4, 5
FAKE = 0x100000  # aligned, never dereferenced
BIG = 1 << 40
BF16, F32 = comba.COMBA_BF16, comba.COMBA_F32


def _struct(cls, **over):
    host = over.pop("host", None)
    s = cls(**over)
    if host is not None:
        a = np.asarray(host, np.int32)
        s.cu_seqlens_host = a.ctypes.data
        s._keep = a
    return s


def conv(**over):
    base = dict(B=2, T=10, D=32, K=4, num_seqs=2, in_dtype=BF16, activation=1)
    return _struct(comba.CombaConvShape, **dict(base, **over))


def select(**over):
    base = dict(B=2, T=10, D=32, N=16, G=1, num_seqs=2, in_dtype=BF16, delta_softplus=1)
    return _struct(comba.CombaSelectShape, **dict(base, **over))


def norm(**over):
    base = dict(rows=5, C=64, G=4, x_dtype=BF16, out_dtype=BF16, activation=1, eps=1e-5)
    return _struct(comba.CombaGroupNormShape, **dict(base, **over))


CALLS = {
    "comba_conv_fwd": ("x w bias? h0? y ht?", None),
    "comba_conv_bwd": ("x w bias? h0? dy dht? dx dw dbias dh0? ws", "ws"),
    "comba_conv_step": ("x w bias? state slots? num_slots y", None),
    "comba_select_fwd": ("u delta A B C D? z? bias? h0? y ht? ws", "ws"),
    "comba_select_fwd_save": ("u delta A B C D? z? bias? h0? y ht? ws", "ws"),
    "comba_select_bwd": ("u delta A B C D? z? bias? h0? dy dht? du ddelta dA dB dC dD dz dbias "
                         "dh0? saved saved_bytes ws", "ws"),
    "comba_select_step": ("u delta A B C D? z? bias? state slots? num_slots y", None),
    "comba_group_norm_fwd": ("x w? b? z? y", None),
    "comba_group_norm_bwd": ("x w? b? z? dy dx dz dw? db? ws", "ws"),
}


SIZES = {"num_slots": 4, "saved_bytes": BIG}


def call(name, shp, ws_bytes=BIG, **over):
    names, ws = CALLS[name]
    args = []
    for n in names.split():
        v = over.get(n.rstrip("?"), SIZES.get(n, FAKE))
        args.append(v)
    if ws:
        args.append(ws_bytes)
    return getattr(comba.load_library(), name)(None if shp is None else ctypes.byref(shp), *args,
                                               None)


def shape_of(name, **over):
    if "conv" in name:
        return conv(**(dict(over, T=1) if "step" in name and "T" not in over else over))
    if "select" in name:
        return select(**(dict(over, T=1) if "step" in name and "T" not in over else over))
    return norm(**over)


def test_layer_header_is_exported_and_bound():
    declared = comba.exported_symbols("comba_layer.h")
    assert declared == sorted(list(CALLS) + [
        "comba_conv_workspace_bytes", "comba_select_fwd_workspace_bytes",
        "comba_select_save_bytes", "comba_select_bwd_workspace_bytes",
        "comba_group_norm_workspace_bytes"])
    out = subprocess.run(["nm", "-D", "--defined-only", comba.library_path()],
                         capture_output=True, text=True, check=True).stdout
    exported = {line.split()[-1] for line in out.splitlines() if line.strip()}
    for name in declared:
        assert name in exported, name
        assert getattr(comba.load_library(), name).argtypes is not None, name
    for name in ("comba_conv", "comba_select", "comba_group_norm"):
        assert name in comba.__all__ and callable(getattr(comba, name))


@pytest.mark.parametrize("name", list(CALLS))
def test_required_pointers(name):
    assert call(name, None) == ENULL
    for n in CALLS[name][0].split():
        if n.endswith("?") or n in SIZES:
            continue
        assert call(name, shape_of(name), **{n: None}) == ENULL, n


@pytest.mark.parametrize("name", list(CALLS))
def test_misaligned_pointers(name):
    for n in CALLS[name][0].split():
        n = n.rstrip("?")
        if n in SIZES:
            continue
        bad = FAKE + (128 if n in ("ws", "saved") else 1)
        assert call(name, shape_of(name), **{n: bad}) == EALIGN, n


@pytest.mark.parametrize("over,code", [
    (dict(K=1), ESHAPE), (dict(K=5), ESHAPE), (dict(D=0), ESHAPE), (dict(B=-1), ESHAPE),
    (dict(num_seqs=3), ESHAPE), (dict(in_dtype=7), EDTYPE), (dict(activation=2), ESHAPE),
    (dict(x_row=16), ESHAPE), (dict(x_row=-32), ESHAPE), (dict(cu_seqlens=FAKE), ESHAPE),
    (dict(host=[0, 10]), ESHAPE)])
def test_conv_shapes(over, code):
    for name in ("comba_conv_fwd", "comba_conv_bwd"):
        assert call(name, conv(**over)) == code
    assert comba.load_library().comba_conv_workspace_bytes(ctypes.byref(conv(**over))) == 0


@pytest.mark.parametrize("over,code", [
    (dict(N=4), ESHAPE), (dict(N=64), ESHAPE), (dict(N=12), ESHAPE), (dict(G=3), ESHAPE),
    (dict(G=0), ESHAPE), (dict(D=0), ESHAPE), (dict(num_seqs=1), ESHAPE), (dict(in_dtype=2), EDTYPE),
    (dict(u_row=8), ESHAPE), (dict(b_row=8), ESHAPE), (dict(c_row=15), ESHAPE),
    (dict(z_row=-1), ESHAPE), (dict(delta_row=31), ESHAPE), (dict(T=-1), ESHAPE)])
def test_select_shapes(over, code):
    for name in ("comba_select_fwd", "comba_select_fwd_save", "comba_select_bwd"):
        assert call(name, select(**over)) == code
    lib = comba.load_library()
    assert lib.comba_select_fwd_workspace_bytes(ctypes.byref(select(**over))) == 0
    assert lib.comba_select_bwd_workspace_bytes(ctypes.byref(select(**over))) == 0
    assert lib.comba_select_save_bytes(ctypes.byref(select(**over))) == 0


@pytest.mark.parametrize("over,code", [
    (dict(G=5), ESHAPE), (dict(G=0), ESHAPE), (dict(C=0), ESHAPE), (dict(rows=-1), ESHAPE),
    (dict(eps=-1.0), ESHAPE), (dict(eps=float("nan")), ESHAPE), (dict(activation=3), ESHAPE),
    (dict(x_dtype=5), EDTYPE), (dict(out_dtype=F32), EDTYPE), (dict(x_row=63), ESHAPE),
    (dict(z_row=-64), ESHAPE)])
def test_norm_shapes(over, code):
    for name in ("comba_group_norm_fwd", "comba_group_norm_bwd"):
        assert call(name, norm(**over)) == code


@pytest.mark.parametrize("host,ok", [([0, 4, 10], True), ([0, 4, 9], False), ([1, 4, 10], False),
                                     ([0, 11, 10], False)])
def test_host_offsets(host, ok):
    """A well-formed table goes on to the next check (a missing output)."""
    want = ENULL if ok else ESHAPE
    assert call("comba_conv_fwd", conv(B=1, cu_seqlens=FAKE, host=host), y=None) == want
    assert call("comba_select_fwd", select(B=1, cu_seqlens=FAKE, host=host), y=None) == want


def test_steps_take_one_token_and_no_offsets():
    for name in ("comba_conv_step", "comba_select_step"):
        assert call(name, shape_of(name, T=2)) == ESHAPE
        assert call(name, shape_of(name, B=1, T=1, cu_seqlens=FAKE, num_seqs=1)) == ESHAPE
        assert call(name, shape_of(name), num_slots=-1) == ESHAPE


def test_workspaces():
    lib = comba.load_library()
    for name, size, shp in (("comba_conv_bwd", lib.comba_conv_workspace_bytes, conv()),
                            ("comba_select_fwd", lib.comba_select_fwd_workspace_bytes, select()),
                            ("comba_select_fwd_save", lib.comba_select_save_bytes, select()),
                            ("comba_select_bwd", lib.comba_select_bwd_workspace_bytes, select()),
                            ("comba_group_norm_bwd", lib.comba_group_norm_workspace_bytes, norm())):
        n = size(ctypes.byref(shp))
        assert n > 0
        assert call(name, shp, ws_bytes=n - 1) == EWS, name
    # the states kept for the backward: one per 48 tokens (8 states a channel: 32) and sequence
    for n, every in ((16, 48), (8, 32)):
        long = select(B=1, T=32000, num_seqs=1, N=n)
        kept = (32000 // every + 2) * 32 * n * 4
        assert lib.comba_select_save_bytes(ctypes.byref(long)) >= kept
        assert call("comba_select_bwd", long, saved_bytes=kept - 1) == EWS
        assert lib.comba_select_bwd_workspace_bytes(ctypes.byref(long)) >= 32000 * 2 * n * 4


def test_tokens_need_a_sequence():
    assert call("comba_conv_fwd", conv(B=1, num_seqs=0, cu_seqlens=FAKE)) == ESHAPE
    assert call("comba_select_fwd", select(B=1, num_seqs=0, cu_seqlens=FAKE)) == ESHAPE


def test_binding_refuses_before_the_library():
    """Host tensors and wrong shapes raise; the row rules are checked on host strides."""
    import torch

    from paper_2506_02475_amd.layer import _row

    x = torch.zeros(2, 3, 8)
    with pytest.raises(comba.CombaError, match="GPU"):
        comba.comba_conv_fwd(x, torch.zeros(8, 4))
    with pytest.raises(comba.CombaError, match="GPU"):
        comba.comba_select_fwd(x, x, torch.zeros(8, 16), x, x)
    with pytest.raises(comba.CombaError, match="GPU"):
        comba.comba_group_norm_fwd(x, 2)
    f, dev = torch.float32, -1
    wide = torch.zeros(2, 3, 20)
    assert _row("x", x, 2, (2, 3, 8), f, dev) == 0
    assert _row("x", wide[..., 4:12], 2, (2, 3, 8), f, dev) == 20
    assert _row("x", wide[:, :1, 4:12], 2, (2, 1, 8), f, dev) == 60
    assert _row("x", wide[:1, :, 4:12], 2, (1, 3, 8), f, dev) == 20
    assert _row("b", wide[..., 4:12].unflatten(-1, (2, 4)), 2, (2, 3, 2, 4), f, dev) == 20
    for bad in (wide[..., ::2][..., :8], wide[:, :2, :8], wide[:, ::2, :8],
                torch.zeros(2, 1, 8).expand(2, 3, 8), torch.zeros(2, 8, 3).transpose(1, 2)):
        with pytest.raises(comba.CombaError, match="x"):
            _row("x", bad, 2, tuple(bad.shape), f, dev)


FAR = 1 << 23  # elements between rows: one token of each of a batch's long rows


@pytest.mark.parametrize("name,rows", [
    ("comba_conv_fwd", ("x_row",)), ("comba_conv_step", ("x_row",)),
    ("comba_select_step", ("u_row", "delta_row", "z_row", "b_row", "c_row")),
    ("comba_group_norm_fwd", ("x_row", "z_row"))])
def test_rows_far_apart_are_taken(name, rows):
    """They go on to the next check (a missing output); spans past 64-bit offsets do not."""
    for r in rows:
        assert call(name, shape_of(name, **{r: FAR}), y=None) == ENULL, r
        assert call(name, shape_of(name, **{r: (1 << 57) // 10}), y=None) == ENULL, r
        assert call(name, shape_of(name, **{r: 1 << 60}), y=None) == ESHAPE, r


def test_the_scan_states_the_limit_of_its_rows():
    """Its tiles address rows by 32-bit offsets: rows up to 2^22 elements apart, refused by
    name above that."""
    import torch

    for r in ("u_row", "delta_row", "z_row", "b_row", "c_row"):
        for name in ("comba_select_fwd", "comba_select_fwd_save", "comba_select_bwd"):
            assert call(name, select(**{r: FAR})) == ESHAPE, (name, r)
            missing = {"dA": None} if name.endswith("bwd") else {"y": None}
            assert call(name, select(**{r: 1 << 22}), **missing) == ENULL, (name, r)
    from paper_2506_02475_amd.layer import _row

    far = torch.empty_strided((2, 1, 8), (FAR, FAR, 1), device="meta")
    dev = far.get_device()
    assert _row("z", far, 2, (2, 1, 8), torch.float32, dev) == FAR
    with pytest.raises(comba.CombaError, match="rows of z .*4194304"):
        _row("z", far, 2, (2, 1, 8), torch.float32, dev, 1 << 22)


def test_a_workspace_has_to_be_device_memory():
    """Host memory, or fewer bytes behind a view than it has elements, would be written past."""
    import torch

    from paper_2506_02475_amd.layer import _workspace

    def size(shp):
        return 1000

    host = torch.empty(2000, dtype=torch.uint8)
    with pytest.raises(comba.CombaError, match="workspace"):
        _workspace(size, b"", host, torch.device("cuda", 0))
    meta = torch.device("meta")
    assert _workspace(size, b"", None, meta).numel() == 1000
    small = torch.empty(999, dtype=torch.uint8, device=meta)
    assert _workspace(size, b"", small, meta).numel() == 1000  # too small: made anew
    good = torch.empty(1000, dtype=torch.uint8, device=meta)
    assert _workspace(size, b"", good, meta) is good
    with pytest.raises(comba.CombaError, match="workspace"):
        _workspace(size, b"", good[:1].expand(5000), meta)


def test_another_stream_waits_for_the_current_one(monkeypatch):
    """What a call makes comes from the current stream's memory, whose last users may still be
    at work there: a stream given by handle has to wait for them before it writes."""
    import torch

    from paper_2506_02475_amd import layer

    log = []

    class Stream:
        def __init__(self, handle, device=None):
            self.handle = handle

        def wait_stream(self, other):
            log.append((self.handle, "waits for", other.handle))

    class Made:
        def record_stream(self, s):
            log.append(("used on", s.handle))

    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 7, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: Stream(7))
    assert layer._on(None, 0, Made()) == 7 and layer._on(7, 0, Made()) == 7
    assert log == []
    assert layer._on(9, 0, Made(), None) == 9
    assert log == [(9, "waits for", 7), ("used on", 9)]
    # handle 0 is the default stream
    monkeypatch.setattr(torch.cuda, "default_stream", lambda dev=None: Stream("default"))
    del log[:]
    assert layer._on(0, 0, Made()) == 0
    assert log == [("default", "waits for", 7), ("used on", "default")]


def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    """Their default stream has the handle of the current device's, so the kernels would run
    on the wrong GPU, with pointers of the other."""
    import torch

    from paper_2506_02475_amd import layer

    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    assert layer._on(None, 0) == 0
    with pytest.raises(comba.CombaError, match="device 1.*current"):
        layer._on(None, 1)


def test_a_scan_of_more_workgroups_than_a_launch_holds():
    """A launch has fewer than 2^32 threads: more sequences x channel blocks are refused before
    the first of a call's launches, not by one of them."""
    lib = comba.load_library()
    for N, most in ((8, 2 ** 23 - 1), (16, (2 ** 32 - 1) // 768), (32, (2 ** 32 - 1) // 768)):
        for S, fits in ((most, True), (most + 1, False)):
            shp = select(B=S, num_seqs=S, T=1, D=512 // N, N=N)
            assert call("comba_select_fwd", shp, y=None) == (ENULL if fits else ESHAPE), (N, S)
            assert call("comba_select_bwd", shp, dA=None) == (ENULL if fits else ESHAPE), (N, S)
            assert (lib.comba_select_save_bytes(ctypes.byref(shp)) > 0) == fits
    S = 1 << 23  # the steps take several rows a thread
    assert call("comba_select_step", select(B=S, num_seqs=S, T=1, D=32), y=None) == ENULL
