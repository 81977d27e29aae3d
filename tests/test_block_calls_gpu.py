"""How a block's operators behave as calls: autograd, differences, bits, non-finite values,
offsets, streams and graphs."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _inputs(T=300, H=4, Hk=2, dk=64, dv=48, B=2, dtype=None, seed=0, states=None):
    import torch

    dtype = dtype or torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rnd(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    q, k, v = (rnd(B, T, h, d).to(dtype) * d ** -0.25 for h, d in ((H, dk), (Hk, dk), (H, dv)))
    g = (-torch.rand(B, T, H, device="cuda", generator=gen) / 10).to(dtype)
    return [q, k, v, g, 0.3 * rnd(B if states is None else states, H, dk, dv)]


def _norm_inputs(rows=200, C=640, seed=1):
    import torch

    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rnd(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    y, z = rnd(rows, C).bfloat16(), rnd(rows, C).bfloat16()
    return y, rnd(rows, C), 1 + 0.1 * rnd(C), dict(post_weight=1 + 0.1 * rnd(C), z=z,
                                                   scale=0.5 + 0.1 * rnd(C))


def test_autograd_gives_the_direct_calls_gradients():
    import torch

    import paper_2506_02475_amd as comba

    ins = _inputs()
    leaves = [t.clone().requires_grad_() for t in ins]
    o, ht = comba.comba_decay(*leaves)
    do, dht = torch.randn_like(o), torch.randn_like(ht)
    torch.autograd.backward([o, ht], [do, dht])
    o2, ht2, ws = comba.comba_decay_fwd_save(*ins)
    gr = comba.comba_decay_bwd(*ins, do, dht, workspace=ws)
    assert torch.equal(o, o2) and torch.equal(ht, ht2)
    for t, n in zip(leaves, ("dq", "dk", "dv", "dg", "dh0")):
        assert torch.equal(t.grad, gr[n]), n
    # the final state alone
    leaves = [t.clone().requires_grad_() for t in ins]
    comba.comba_decay(*leaves)[1].backward(dht)
    gr = comba.comba_decay_bwd(*ins, torch.zeros_like(o), dht, workspace=ws)
    for t, n in zip(leaves, ("dq", "dk", "dv", "dg", "dh0")):
        assert torch.equal(t.grad, gr[n]), n

    y, x, w, kw = _norm_inputs()
    leaf = {n: t.clone().requires_grad_() for n, t in dict(kw, y=y, x=x, w=w).items()}
    r, n = comba.comba_block_norm(leaf["y"], leaf["x"], leaf["w"], **{k: leaf[k] for k in kw})
    dr, dn = torch.randn_like(r), torch.randn_like(n)
    torch.autograd.backward([r, n], [dr, dn])
    gr = comba.comba_block_norm_bwd(y, x, w, dr, dn, **kw)
    for a, b in (("y", "dy"), ("x", "dx"), ("w", "dweight"), ("post_weight", "dpost_weight"),
                 ("z", "dz"), ("scale", "dscale")):
        assert torch.equal(leaf[a].grad, gr[b]), a


def test_gradients_by_differences():
    """fp32: the outputs' directional central difference against the gradients.  A step of 2^-6
    of unit directions: the second-order term (third derivatives of products of three factors)
    about 2^-12, rounding 1e-6 of the loss's terms over 2^-5, 3e-5."""
    import torch

    import paper_2506_02475_amd as comba

    ins = _inputs(T=150, dk=40, dv=24, dtype=torch.float32)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    o, ht, ws = comba.comba_decay_fwd_save(*ins)
    do, dht = (torch.randn(t.shape, device="cuda", generator=gen) for t in (o, ht))
    gr = comba.comba_decay_bwd(*ins, do, dht, workspace=ws)

    def loss(args):
        a, b = comba.comba_decay_fwd(*args)
        return ((a.double() * do).sum() + (b.double() * dht).sum()).item()

    e = 2.0 ** -6
    for i, n in enumerate(("dq", "dk", "dv", "dg", "dh0")):
        d = torch.randn(ins[i].shape, device="cuda", generator=gen) * (0.01 if n == "dg" else 1.0)
        up, dn = list(ins), list(ins)
        up[i], dn[i] = ins[i] + e * d, ins[i] - e * d
        num, ana = (loss(up) - loss(dn)) / (2 * e), (gr[n].double() * d).sum().item()
        size = (gr[n].double() * d).norm().item()
        assert abs(num - ana) <= 1e-3 * (abs(ana) + size), (n, num, ana)


def test_two_calls_give_the_same_bits():
    import torch

    import paper_2506_02475_amd as comba

    ins = _inputs(T=1500, B=1, H=2, Hk=1)  # in segments
    do = torch.randn(1, 1500, 2, 48, device="cuda").bfloat16()
    outs = []
    for _ in range(2):
        o, ht, ws = comba.comba_decay_fwd_save(*ins)
        gr = comba.comba_decay_bwd(*ins, do, workspace=ws)
        outs.append([o, ht] + [gr[n] for n in sorted(gr)])
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_host_offsets_change_no_result():
    import torch

    import paper_2506_02475_amd as comba

    lens = [5, 700, 0, 300, 64]
    cu = np.cumsum([0] + lens).astype(np.int32)
    ins = _inputs(T=sum(lens), B=1, states=len(lens), H=2, Hk=2)
    dev = torch.from_numpy(cu).cuda()
    a = comba.comba_decay_fwd(*ins, cu_seqlens=dev, cu_seqlens_host=cu)
    b = comba.comba_decay_fwd(*ins, cu_seqlens=dev)
    for x, y in zip(a, b):
        assert torch.allclose(x.float(), y.float(), rtol=2.0 ** -7, atol=1e-5)


def test_non_finite_values_stay_in_their_sequence_and_head():
    """And reach no row of their own more than 63 before them (gradients: behind them)."""
    import torch

    import paper_2506_02475_amd as comba

    lens = [40, 270, 33, 64]
    cu = torch.tensor(np.cumsum([0] + lens), dtype=torch.int32, device="cuda")
    q, k, v, g, h0 = _inputs(T=sum(lens), B=1, H=4, Hk=4, states=4)
    do = torch.randn(1, sum(lens), 4, 48, device="cuda").bfloat16()

    def run(q, k, v, g):
        o, ht, ws = comba.comba_decay_fwd_save(q, k, v, g, h0, cu_seqlens=cu)
        gr = comba.comba_decay_bwd(q, k, v, g, h0, do, workspace=ws, cu_seqlens=cu)
        return dict(gr, o=o, ht=ht)

    clean = run(q, k, v, g)
    for name in ("q", "k", "v", "g"):
        args = dict(q=q.clone(), k=k.clone(), v=v.clone(), g=g.clone())
        args[name][0, 40 + 200, 1] = float("nan")  # sequence 1, head 1
        got = run(**args)
        for n in ("o", "dq", "dk", "dv", "dg"):
            a, b = got[n][0], clean[n][0]
            for s, e in ((0, 40), (310, 407)):
                assert torch.equal(a[s:e], b[s:e]), (name, n)
            for h in (0, 2, 3):
                assert torch.equal(a[:, h], b[:, h]), (name, n)
        others = [0, 2, 3]
        assert torch.equal(got["ht"][others], clean["ht"][others])
        assert torch.equal(got["o"][0, 40:40 + 137], clean["o"][0, 40:40 + 137]), name
        assert not torch.isfinite(got["o"][0, 240, 1]).any(), name
        if name != "q":
            assert not torch.isfinite(got["ht"][1, 1]).all(), name


def test_malformed_device_offsets_stay_in_bounds():
    import torch

    import paper_2506_02475_amd as comba

    ins = _inputs(T=90, B=1, states=3, H=2, Hk=1)
    do = torch.randn(1, 90, 2, 48, device="cuda").bfloat16()
    for bad in ([-5, 60, 10, 4000], [90, 90, 0, 0], [0, 2 ** 31 - 1, -2 ** 31, 90]):
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        o, ht, ws = comba.comba_decay_fwd_save(*ins, cu_seqlens=cu)
        comba.comba_decay_bwd(*ins, do, workspace=ws, cu_seqlens=cu)
        torch.cuda.synchronize()


@pytest.mark.parametrize("Hk", [2, 1])
def test_rows_behind_the_last_sequence_are_left(monkeypatch, Hk):
    import torch

    import paper_2506_02475_amd as comba
    from paper_2506_02475_amd import block

    ins = _inputs(T=200, B=1, states=2, H=2, Hk=Hk)
    cu = torch.tensor([0, 70, 133], dtype=torch.int32, device="cuda")

    def filled(v, H):
        return torch.full(v.shape[:2] + (H, v.shape[-1]), 7.0, device="cuda", dtype=v.dtype)

    monkeypatch.setattr(block, "_outputs", filled)
    monkeypatch.setattr(block, "_like", lambda t, dtype=None: torch.full_like(t, 7.0))
    o, ht, ws = comba.comba_decay_fwd_save(*ins, cu_seqlens=cu)
    do = torch.randn(1, 200, 2, 48, device="cuda").bfloat16()
    gr = comba.comba_decay_bwd(*ins, do, workspace=ws, cu_seqlens=cu)
    for n, t in dict(gr, o=o).items():
        if n != "dh0":
            assert bool((t[:, 133:] == 7.0).all()), n
            assert not bool((t[:, :133] == 7.0).all()), n


def _calls(s):
    """Every call on stream s, its temporary memory reused by the current stream right after."""
    import torch

    import paper_2506_02475_amd as comba

    ins = _inputs(T=900, B=1, H=2, Hk=1)
    do = torch.ones(1, 900, 2, 48, device="cuda").bfloat16()
    y, x, w, kw = _norm_inputs()
    pool = ins[4].repeat(5, 1, 1, 1)
    o, ht, ws = comba.comba_decay_fwd_save(*ins, stream=s)
    gr = comba.comba_decay_bwd(*ins, do, ht, workspace=ws, stream=s)
    out = [o, ht] + [gr[n] for n in sorted(gr)]
    out += list(comba.comba_decay_fwd(*ins, stream=s))
    out += [comba.comba_decay_step(*(t[0, :5] for t in ins[:4]), pool, stream=s), pool]
    r, n = comba.comba_block_norm_fwd(y, x, w, stream=s, **kw)
    gr = comba.comba_block_norm_bwd(y, x, w, r, n, stream=s, **kw)
    out += [r, n] + [gr[k] for k in sorted(gr)]
    del ws
    for _ in range(8):  # the current stream takes what was freed
        torch.full((1 << 20,), float("nan"), device="cuda")
    return out


def test_a_stream_given_by_handle():
    import torch

    want = _calls(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = _calls(side.cuda_stream)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def test_captured_steps_and_training_follow_new_inputs():
    """Two graphs (a step in place; forwards and backwards by the direct calls), replayed in
    turn with eager work between the replays."""
    import torch

    import paper_2506_02475_amd as comba

    q, k, v, g, h0 = _inputs(T=6, B=3)
    y, x, w, kw = _norm_inputs(rows=3, C=4 * 48)
    pool = torch.zeros_like(h0)
    token = [t[:, 0].clone() for t in (q, k, v, g)]

    def step(pool):
        o = comba.comba_decay_step(*token, pool)
        return comba.comba_block_norm_fwd(o.flatten(1), x, w, **kw)

    big = _inputs(T=700, B=1, H=2, Hk=1, seed=5)
    do = torch.randn(1, 700, 2, 48, device="cuda").bfloat16()

    def train():
        o, ht, ws = comba.comba_decay_fwd_save(*big)
        gr = comba.comba_decay_bwd(*big, do, workspace=ws)
        r, n = comba.comba_block_norm_fwd(y, x, w, **kw)
        gn = comba.comba_block_norm_bwd(y, x, w, r, n, **kw)
        return [o, ht, r, n] + [gr[a] for a in sorted(gr)] + [gn[a] for a in sorted(gn)]

    step(pool.clone()), train()
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        out1 = step(pool)
    with torch.cuda.graph(g2):
        out2 = train()
    pool.copy_(h0)
    eager = h0.clone()
    for i in range(5):
        for t, s in zip(token, (q, k, v, g)):
            t.copy_(s[:, i])
        big[0].mul_(-1.0)
        y.add_(0.25)
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out1] + [pool.clone()] + [t.clone() for t in out2]
        want = list(step(eager)) + [eager] + train()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (i, n)


def test_steps_continue_a_prompt():
    """The states of a prompt's call, and tokens one by one, give the whole call's outputs."""
    import torch

    import paper_2506_02475_amd as comba

    ins = _inputs(T=140, B=3, dtype=torch.float32)
    whole, end = comba.comba_decay_fwd(*ins)
    _, state = comba.comba_decay_fwd(*(t[:, :130].contiguous() for t in ins[:4]), ins[4])
    for t in range(130, 140):
        o = comba.comba_decay_step(*(x[:, t] for x in ins[:4]), state)
        assert (o - whole[:, t]).abs().max() <= 1e-5 * whole.abs().max()
    assert (state - end).abs().max() <= 1e-5 * end.abs().max()


def _far_rows(t, row, offset):
    """t [1,T,..] as a column slice of rows ``row`` elements apart, at ``offset`` in each; what
    lies between is not written."""
    import torch

    wide = torch.empty(t.shape[1] * row, device="cuda", dtype=t.dtype)
    far = wide.view(1, t.shape[1], row)[..., offset:offset + t[0, 0].numel()]
    far = far.unflatten(-1, t.shape[2:])
    far.copy_(t)
    return far


def test_offsets_past_32_bits():
    """Rows at the farthest distance that is taken, and a pool of states over 2^31 elements: the
    bits of the same call on contiguous memory."""
    import torch

    import paper_2506_02475_amd as comba

    q, k, v, g, _ = _inputs(T=600, H=2, Hk=2, dk=64, dv=64, B=1)
    row = 1 << 22
    assert q.shape[1] * row > 1 << 31
    do = v.clone()

    def run(q, g):
        o, ht, ws = comba.comba_decay_fwd_save(q, k, v, g)
        return [o, ht] + [x for x in comba.comba_decay_bwd(q, k, v, g, None, do, workspace=ws,
                                                           need_dh0=False).values()
                          if x is not None]

    want = run(q, g)
    for far_q, far_g in ((_far_rows(q, row, 64), g), (q, _far_rows(g, row, 8))):
        for a, b in zip(run(far_q, far_g), want):
            assert torch.equal(a, b)
        del far_q, far_g
    H, d = 2, 256
    slots = (1 << 31) // (H * d * d) + 2
    pool = torch.empty(slots, H, d, d, device="cuda")
    q1, k1, v1, g1 = (torch.randn(2, *s, device="cuda").bfloat16()
                      for s in ((H, d), (H, d), (H, d), (H,)))
    g1 = -g1.abs()
    small = torch.randn(2, H, d, d, device="cuda")
    at = torch.tensor([slots - 1, 0], device="cuda", dtype=torch.int32)
    pool[at.long()] = small
    o = comba.comba_decay_step(q1, k1, v1, g1, pool, slots=at)
    want = comba.comba_decay_step(q1, k1, v1, g1, small)
    assert torch.equal(o, want) and torch.equal(pool[at.long()], small)


def test_norm_rows_past_32_bits():
    import torch

    import paper_2506_02475_amd as comba

    y, x, w, kw = _norm_inputs(rows=600, C=640)
    row = 1 << 22
    far = _far_rows(y[None], row, 64)[0]
    want = comba.comba_block_norm_fwd(y, x, w, **kw)
    got = comba.comba_block_norm_fwd(far, x, w, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    gr = [comba.comba_block_norm_bwd(t, x, w, x, y, **kw) for t in (y, far)]
    assert all(torch.equal(gr[0][n], gr[1][n]) for n in gr[0])
