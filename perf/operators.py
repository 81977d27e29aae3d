"""Performance cases of the layer operators around a recurrent token mixer: the
short causal convolution with its history, the selective state space scan, and
the group norm per token with an activation or a gate.

Each case is one call of an operator (or its forward and backward) as a program
that serves or trains such a layer makes it.  Widths are those of this
repository's layers (16 heads of 128 = 2,048 channels, twice that for an
expanded inner width), row lengths and packed batches those of its workloads,
and ragged sizes around them.  A layer's projections leave slices: z, B and C
come as column slices of a wider row, as the layer has them.

A case is a dict of plain values:
  op      conv | scan | norm
  kind    step (one token per sequence, states in slots, in place) | fwd | train
  B, T    rows and tokens per row (packed: B = 1, T the total)
  lens    packed sequence lengths "n,n,..." or ""
  D       channels
  N, G    scan: states per channel and B/C groups; norm: G groups (N = 0)
  K       conv: taps
  dtype   bf16 | f32 of the activations
  h0      initial states given (norm: x arrives in fp32, as from comba_chunk_fwd)
  z       gated
"""
import math

import torch

own = False


def _case(op, kind, B, T, D, *, lens=(), N=0, G=1, K=0, dtype="bf16", h0=False, z=True, name=None):
    c = {"op": op, "kind": kind, "B": B, "T": sum(lens) if lens else T, "D": D,
         "lens": ",".join(str(n) for n in lens), "N": N, "G": G, "K": K, "dtype": dtype,
         "h0": h0, "z": z}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # A serving batch's step: the convolution of 64 sequences' next tokens.
        _case("conv", "step", 64, 1, 4096, K=4, h0=True, name="conv_step_b64"),
        # Packed prompts that continue cached sequences, one of a single token.
        _case("conv", "fwd", 1, 0, 2048, K=4, h0=True,
              lens=(3001, 517, 64, 4096, 1250, 777, 2048, 1, 2900, 1730), name="conv_prompt_16k"),
        # Pretraining step of a layer of the expanded width: forward and backward.
        _case("conv", "train", 4, 4096, 4096, K=4, name="conv_train_b4_t4096"),
        # One user's chat: one token of one sequence.
        _case("scan", "step", 1, 1, 2048, N=16, h0=True, name="scan_step_b1"),
        # A large serving batch's step.
        _case("scan", "step", 200, 1, 4096, N=16, h0=True, name="scan_step_b200"),
        # One prompt of ordinary length (not a multiple of anything) before decoding.
        _case("scan", "fwd", 1, 1000, 2048, N=16, name="scan_prompt_b1_t1000"),
        # Packed prompts of unequal length, with cached states.
        _case("scan", "fwd", 1, 0, 2048, N=16, h0=True,
              lens=(8000, 517, 64, 4096, 1250, 15777, 2048, 1, 2900, 1730), name="scan_prompt_36k"),
        # Full-precision run of a small odd-sized model: forward and gradients.
        _case("scan", "train", 2, 777, 1000, N=8, G=2, dtype="f32", h0=True, name="scan_train_f32"),
        # Pretraining step of a layer of the expanded width: forward and backward.
        _case("scan", "train", 4, 4096, 4096, N=16, name="scan_train_b4_t4096"),
        # A serving batch's step: the norm of 64 tokens' heads, gated.
        _case("norm", "fwd", 64, 1, 2048, G=16, h0=True, name="norm_step_b64"),
        # A batch of prompts: the mixer's fp32 output, normed per head of 256 and gated.
        _case("norm", "fwd", 4, 4096, 2048, G=8, h0=True, name="norm_prompt_b4_t4096"),
        # Pretraining step: forward and backward at the expanded width.
        _case("norm", "train", 4, 4096, 4096, G=32, name="norm_train_b4_t4096"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo=256, hi=4096):
    """Channels: mostly multiples of 64, now and then any number."""
    d = _log_int(rng, lo, hi)
    d = d if rng.random() < 0.2 else max(64, d // 64 * 64)
    return 3008 if d == 3072 else d


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    D, z = _width(rng), rng.random() < 0.7
    room = 4 * 4096 * 4096 // (2 if dtype == "f32" else 1)  # tokens x channels at most
    kinds = ["fwd", "train"] if op == "norm" else ["step", "fwd", "train"]
    kind = rng.choice(kinds)
    N, G, K = 0, 1, 0
    if op == "conv":
        K, z = rng.choice([2, 3, 4, 4]), False
    if op == "scan":
        N = rng.choice([8, 16, 16, 16, 32])
        G = rng.choice([1, 1, 2]) if D % 2 == 0 else 1
        room = room * 16 // max(N, 16) // 2
    if op == "norm":
        size = rng.choice([64, 64, 128, 128, 256, 96, 100])
        G = max(1, D // size)
        D = G * size
        D = D - size if D == 3072 else D
        G = D // size
    if kind == "step":
        return _case(op, kind, _log_int(rng, 1, 256), 1, D, N=N, G=G, K=K, dtype=dtype, h0=True,
                     z=z)
    h0 = rng.random() < 0.5
    form = rng.choice(["batch", "one", "packed"])
    if form == "packed" and op != "norm":
        n = rng.randint(2, 20)
        lens = [_log_int(rng, 1, max(2, min(16384, room // D // n))) for _ in range(n)]
        return _case(op, kind, 1, 0, D, lens=lens, N=N, G=G, K=K, dtype=dtype, h0=h0, z=z)
    B = 1 if form == "one" else _log_int(rng, 1, 16)
    T = _log_int(rng, 16, max(32, min(16384, room // D // B)))
    return _case(op, kind, B, T, D, N=N, G=G, K=K, dtype=dtype, h0=h0, z=z)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens(case):
    return [int(x) for x in case["lens"].split(",")] if case["lens"] else []


def prepare(case, seed):
    """Seeded inputs in their storage types, with the layer's distributions: activations
    of unit size, decay rates -1..-N with noise, steps of 0.001 to 0.1 behind the softplus."""
    dev, dt, f32 = torch.device("cuda"), _dtype(case), torch.float32
    gen = torch.Generator(device=dev)
    gen.manual_seed(1000003 * int(seed) + 29)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=f32)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=dev, dtype=f32)

    B, T, D, N, G, K = (case[n] for n in ("B", "T", "D", "N", "G", "K"))
    s = {"op": case["op"], "kind": case["kind"], "G": G, "packed": {}, "starts": None, "rows": B}
    lens = _lens(case)
    if lens:
        cu = torch.zeros(len(lens) + 1, dtype=torch.int32)
        cu[1:] = torch.cumsum(torch.tensor(lens), 0)
        s["packed"] = {"cu_seqlens": cu.to(dev), "cu_seqlens_host": cu.numpy()}
        s["starts"] = cu.to(dev).long()
        s["rows"] = len(lens)
    S = s["rows"]
    step = case["kind"] == "step"
    lead = (B,) if step else (B, T)
    if step:  # the batch's states lie anywhere in the server's pool
        s["slots"] = torch.randperm(S + S // 4 + 1, generator=gen, device=dev)[:S].int()
        S = S + S // 4 + 1
    xz = normal(*lead, 2 * D).to(dt)  # the input projection: x, z side by side
    if case["op"] == "conv":
        s["x"] = xz[..., :D]
        s["w"], s["b"] = normal(D, K) / K ** 0.5, 0.1 * normal(D)
        s["h0"] = normal(S, K - 1, D).to(dt) if case["h0"] else None
        s["dy"] = normal(B, T, D).to(dt)
    elif case["op"] == "scan":
        R = max(1, D // 32)
        bc = normal(*lead, R + 2 * G * N).to(dt)  # the second projection: delta's rank, B, C
        s["B"] = bc[..., R:R + G * N].unflatten(-1, (G, N))
        s["C"] = bc[..., R + G * N:].unflatten(-1, (G, N))
        x = normal(*lead, D)
        s["u"] = (x * torch.sigmoid(x)).to(dt)
        s["delta"] = (0.5 * normal(*lead, D)).to(dt)
        s["A"] = -torch.arange(1, N + 1, device=dev, dtype=f32) * torch.exp(0.1 * normal(D, N))
        tau = torch.exp(math.log(0.001) + math.log(100.0) * uniform(D))
        s["bias"] = tau + torch.log(-torch.expm1(-tau))  # softplus(bias) = tau
        s["D"] = 1 + 0.1 * normal(D)
        s["z"] = xz[..., D:] if case["z"] else None
        s["h0"] = 0.1 * normal(S, D, N) if case["h0"] else None
        s["dy"] = normal(B, T, D).to(dt)
    else:
        s["x"] = 0.5 * normal(B, T, D) + 0.1 if case["h0"] else (0.5 * normal(B, T, D) + 0.1).to(dt)
        s["out"] = dt
        s["w"], s["b"] = 1 + 0.1 * normal(D), 0.1 * normal(D)
        s["z"] = xz[..., D:] if case["z"] else None
        s["dy"] = normal(B, T, D).to(dt)
    return s


# ---------------------------------------------------------------------------
# the plain forms: elementary operations in 32 bits, rounded once at the end
# ---------------------------------------------------------------------------
def _f(x):
    return None if x is None else x.float()


def _first(s, T, device):
    """Each sequence's first token, the token after its last, and whether it has any."""
    B = 1 if s["starts"] is not None else s["rows"]
    at = s["starts"] if s["starts"] is not None else torch.arange(B + 1, device=device) * T
    a, b = at[:-1], at[1:]
    live = b > a
    return a, b, live


def _history(s, x, K):
    """The K - 1 inputs before every token, [tokens, K - 1, D], and the extended input's
    row of each: rows of h0 (or zeros) before a sequence's first token."""
    B, T, D = x.shape
    a, b, _ = _first(s, T, x.device)
    n = B * T
    tok = torch.arange(n, device=x.device)
    seq = torch.bucketize(tok, b, right=True)
    h0 = torch.zeros(len(a), K - 1, D, device=x.device) if s["h0"] is None else s["h0"].float()
    pool = torch.cat([h0.reshape(-1, D), x.float().reshape(n, D)])  # [S (K - 1) + tokens, D]
    off = torch.arange(K, device=x.device) - (K - 1)
    rel = tok[:, None] + off - a[seq][:, None]  # position in the sequence, negative: history
    src = torch.where(rel >= 0, len(a) * (K - 1) + tok[:, None] + off,
                      seq[:, None] * (K - 1) + (K - 1) + rel)
    tail = b[:, None] + off[1:] - 1  # the last K - 1 rows of each extended sequence
    trel = tail - a[:, None]
    s_at = torch.arange(len(a), device=x.device)[:, None]
    tsrc = torch.where(trel >= 0, len(a) * (K - 1) + tail, s_at * (K - 1) + (K - 1) + trel)
    return pool, src, tsrc


def _plain_conv(s):
    x, w, b = s["x"], s["w"], s["b"]
    D, K = w.shape
    if s["kind"] == "step":
        at = s["slots"].long()
        win = torch.cat([s["h0"][at].float(), x.float()[:, None]], 1)  # [B, K, D]
        u = (win * w.t()).sum(1) + b
        s["h0"][at] = win[:, 1:].to(x.dtype)
        return {"y": (u * torch.sigmoid(u)).to(x.dtype), "state": s["h0"]}
    pool, src, tail = _history(s, x, K)
    win = pool[src]  # [tokens, K, D]
    u = (win * w.t()).sum(1) + b
    sg = torch.sigmoid(u)
    out = {"y": (u * sg).to(x.dtype).reshape(x.shape), "ht": pool[tail].to(x.dtype)}
    if s["kind"] == "train":
        du = s["dy"].float().reshape(-1, D) * sg * (1 + u * (1 - sg))
        dp = torch.zeros_like(pool)
        dp.index_add_(0, src.reshape(-1), (du[:, None] * w.t()).reshape(-1, D))
        n = len(tail) * (K - 1)
        out["dx"] = dp[n:].to(x.dtype).reshape(x.shape)
        out["dw"] = (du[:, None] * win).sum(0).t()
        out["db"] = du.sum(0)
        out["dh0"] = dp[:n].reshape(-1, K - 1, D).to(x.dtype) if s["h0"] is not None else None
    return {k: v for k, v in out.items() if v is not None}


def _linear_scan(a, x):
    """h_t = a_t h_{t-1} + x_t along dim 1, by doubling."""
    k, T = 1, x.shape[1]
    while k < T:
        x = torch.cat([x[:, :k], torch.addcmul(x[:, k:], a[:, k:], x[:, :-k])], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1) if 2 * k < T else a
        k *= 2
    return x


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))


def _wide(x, D):
    """[..., G, N] to [..., D, N]: a group's rows for its D / G channels."""
    G, N = x.shape[-2:]
    return x.unsqueeze(-2).expand(x.shape[:-1] + (D // G, N)).reshape(x.shape[:-2] + (D, N))


def _plain_scan(s):
    u, delta, A, skip, z = _f(s["u"]), _f(s["delta"]), s["A"], s["D"], _f(s["z"])
    D, N = A.shape
    Bm, Cm = _wide(_f(s["B"]), D), _wide(_f(s["C"]), D)
    raw = delta + s["bias"]
    dt = _softplus(raw)
    act = None if z is None else z * torch.sigmoid(z)
    if s["kind"] == "step":
        at = s["slots"].long()
        h = torch.exp(dt[..., None] * A) * s["h0"][at] + (dt * u)[..., None] * Bm
        s["h0"][at] = h
        y = (Cm * h).sum(-1) + skip * u
        return {"y": (y if z is None else y * act).to(s["u"].dtype), "state": s["h0"]}
    B, T = u.shape[:2]
    first, last, live = _first(s, T, u.device)
    a = torch.exp(dt[..., None] * A)
    x = (dt * u)[..., None] * Bm
    flat_a, flat_x = a.reshape(B * T, D, N), x.reshape(B * T, D, N)
    h0 = torch.zeros(len(first), D, N, device=u.device) if s["h0"] is None else s["h0"]
    f, e = first[live], (last - 1)[live]
    flat_x[f] += flat_a[f] * h0[live]
    cut = flat_a.clone()
    cut[f] = 0
    h = _linear_scan(cut.reshape(a.shape), flat_x.reshape(a.shape))
    ht = h0.clone()
    ht[live] = h.reshape(B * T, D, N)[e]
    pre = (Cm * h).sum(-1) + skip * u
    out = {"y": (pre if z is None else pre * act).to(s["u"].dtype), "ht": ht}
    if s["kind"] == "fwd":
        return out
    gy = _f(s["dy"])
    if z is not None:
        sg = torch.sigmoid(z)
        out["dz"] = (gy * pre * sg * (1 + z * (1 - sg))).to(s["u"].dtype)
        gy = gy * act
    up = torch.zeros_like(cut)  # the decay towards the token after
    up[:-1] = cut[1:]
    dh = _linear_scan(up.reshape(a.shape).flip(1), (Cm * gy[..., None]).flip(1)).flip(1)
    prev = torch.zeros_like(cut)
    prev[1:] = h.reshape(B * T, D, N)[:-1]
    prev[f] = h0[live]
    p = dh * a * prev.reshape(a.shape)
    db = (dh * Bm).sum(-1)
    G = s["G"]
    out["du"] = (dt * db + skip * gy).to(s["u"].dtype)
    ddelta = ((p * A).sum(-1) + u * db) * torch.sigmoid(raw)
    out["ddelta"] = ddelta.to(s["u"].dtype)
    out["dA"] = (p * dt[..., None]).sum((0, 1))
    out["dB"] = (dh * (dt * u)[..., None]).unflatten(2, (G, D // G)).sum(3).to(s["u"].dtype)
    out["dC"] = (h * gy[..., None]).unflatten(2, (G, D // G)).sum(3).to(s["u"].dtype)
    out["dD"] = (gy * u).sum((0, 1))
    out["dbias"] = ddelta.sum((0, 1))
    if s["h0"] is not None:
        dh0 = torch.zeros_like(h0)
        dh0[live] = (a * dh).reshape(B * T, D, N)[f]
        out["dh0"] = dh0
    return out


def _plain_norm(s):
    x, w, b, z, G = _f(s["x"]), s["w"], s["b"], _f(s["z"]), s["G"]
    xg = x.unflatten(-1, (G, -1))
    c = xg - xg.mean(-1, keepdim=True)
    rstd = torch.rsqrt((c * c).mean(-1, keepdim=True) + 1e-5)
    xh = (c * rstd).flatten(-2)
    n = xh * w + b
    t = n if z is None else z
    sg = torch.sigmoid(t)
    out = {"y": (t * sg if z is None else n * t * sg).to(s["out"])}
    if s["kind"] == "train":
        dy = _f(s["dy"])
        d = sg * (1 + t * (1 - sg))
        dn = dy * d if z is None else dy * t * sg
        if z is not None:
            out["dz"] = (dy * n * d).to(s["out"])
        g = (dn * w).unflatten(-1, (G, -1))
        xr = c * rstd
        out["dx"] = (rstd * (g - g.mean(-1, keepdim=True) - xr * (g * xr).mean(-1, keepdim=True))
                     ).flatten(-2).to(s["x"].dtype)
        out["dw"], out["db"] = (dn * xh).sum((0, 1)), dn.sum((0, 1))
    return out


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _own_conv(s):
    import paper_2506_02475_amd as comba

    if s["kind"] == "step":
        y = comba.comba_conv_step(s["x"], s["w"], s["b"], s["h0"], slots=s["slots"])
        return {"y": y, "state": s["h0"]}
    y, ht = comba.comba_conv_fwd(s["x"], s["w"], s["b"], s["h0"], **s["packed"])
    out = {"y": y, "ht": ht}
    if s["kind"] == "train":
        gr = comba.comba_conv_bwd(s["x"], s["w"], s["b"], s["h0"], s["dy"],
                                  need_dh0=s["h0"] is not None, **s["packed"])
        out.update(dx=gr["dx"], dw=gr["dw"], db=gr["dbias"])
        if s["h0"] is not None:
            out["dh0"] = gr["dh0"]
    return out


def _own_scan(s):
    import paper_2506_02475_amd as comba

    args = (s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"], s["bias"], s["h0"])
    if s["kind"] == "step":
        return {"y": comba.comba_select_step(*args, slots=s["slots"]), "state": s["h0"]}
    if s["kind"] == "fwd":
        y, ht = comba.comba_select_fwd(*args, **s["packed"])
        return {"y": y, "ht": ht}
    y, ht, ws = comba.comba_select_fwd_save(*args, **s["packed"])
    gr = comba.comba_select_bwd(*args, s["dy"], workspace=ws, need_dh0=s["h0"] is not None,
                                **s["packed"])
    out = {"y": y, "ht": ht, "dbias": gr["ddelta_bias"]}
    out.update({n: gr[n] for n in ("du", "ddelta", "dA", "dB", "dC", "dD")})
    if s["z"] is not None:
        out["dz"] = gr["dz"]
    if s["h0"] is not None:
        out["dh0"] = gr["dh0"]
    return out


def _own_norm(s):
    import paper_2506_02475_amd as comba

    out = {"y": comba.comba_group_norm_fwd(s["x"], s["G"], s["w"], s["b"], s["z"],
                                           out_dtype=s["out"])}
    if s["kind"] == "train":
        gr = comba.comba_group_norm_bwd(s["x"], s["G"], s["w"], s["b"], s["z"], s["dy"])
        out.update(dx=gr["dx"], dw=gr["dweight"], db=gr["dbias"])
        if s["z"] is not None:
            out["dz"] = gr["dz"]
    return out


def run(s):
    if own:
        return {"conv": _own_conv, "scan": _own_scan, "norm": _own_norm}[s["op"]](s)
    return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}[s["op"]](s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    B, T, D, N, G, K = (case[n] for n in ("B", "T", "D", "N", "G", "K"))
    e = 2 if case["dtype"] == "bf16" else 4
    tok, gate = B * T * D, 1 if case["z"] else 0
    S = len(_lens(case)) or B
    train = case["kind"] == "train"
    if case["op"] == "conv":
        state = S * (K - 1) * D * e
        nbytes = 2 * tok * e + D * (K + 1) * 4 + state + (state if case["h0"] else 0)
        flops = tok * (2 * K + 6)
        if train:  # x and dy in, dx out
            nbytes += 3 * tok * e + 2 * D * (K + 1) * 4 + (2 * state if case["h0"] else 0)
            flops += tok * (6 * K + 14)
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "scan":
        state = S * D * N * 4
        bc = 2 * B * T * G * N * e
        params = D * (N + 2) * 4
        nbytes = tok * e * (3 + gate) + bc + params + state + (state if case["h0"] else 0)
        flops = tok * (7 * N + 12 + 6 * gate)  # an exponential counts as one
        if train:  # u, delta, z, dy, B, C in; du, ddelta, dz, dB, dC out
            nbytes += tok * e * (5 + 2 * gate) + 2 * bc + 2 * params + \
                (2 * state if case["h0"] else 0)
            flops += tok * (23 * N + 30 + 12 * gate)
        return {"bytes": nbytes, "flops": flops}
    ex = 4 if case["h0"] else e
    nbytes = tok * (ex + e * (1 + gate)) + 2 * D * 4
    flops = tok * (14 + gate)
    if train:  # x, z, dy in; dx, dz out
        nbytes += tok * (2 * ex + e * (1 + 2 * gate)) + 4 * D * 4
        flops += tok * (28 + 6 * gate)
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------
# the same results in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _spans(case):
    lens = _lens(case) or [case["T"]] * case["B"]
    at, spans = 0, []
    for n in lens:
        spans.append((at, at + n))
        at += n
    return spans


def _exact_conv(case, s):
    K, D = case["K"], case["D"]
    w, b = s["w"].double(), s["b"].double()
    if case["kind"] == "step":
        h = s["h0"].double()
        ext = torch.cat([h[s["slots"].long()], s["x"].double().unsqueeze(1)], 1)
        u = b + sum(w[:, j] * ext[:, j] for j in range(K))
        h[s["slots"].long()] = ext[:, 1:]
        return {"y": u / (1 + torch.exp(-u)), "state": h}
    x, dy = s["x"].double().reshape(-1, D), s["dy"].double().reshape(-1, D)
    parts = {"y": [], "ht": [], "dx": [], "dh0": []}
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    for i, (p, q) in enumerate(_spans(case)):
        n = q - p
        head = torch.zeros(K - 1, D, dtype=x.dtype, device=x.device) if s["h0"] is None \
            else s["h0"][i].double()
        ext = torch.cat([head, x[p:q]])
        u = b + sum(w[:, j] * ext[j:j + n] for j in range(K))
        sg = 1 / (1 + torch.exp(-u))
        parts["y"].append(u * sg)
        parts["ht"].append(ext[n:])
        if case["kind"] == "train":
            du = dy[p:q] * (sg + u * sg * (1 - sg))
            de = torch.zeros_like(ext)
            for j in range(K):
                de[j:j + n] += w[:, j] * du
                dw[:, j] += (du * ext[j:j + n]).sum(0)
            db += du.sum(0)
            parts["dx"].append(de[K - 1:])
            parts["dh0"].append(de[:K - 1])
    out = {"y": torch.cat(parts["y"]).reshape(s["x"].shape), "ht": torch.stack(parts["ht"])}
    if case["kind"] == "train":
        out.update(dx=torch.cat(parts["dx"]).reshape(s["x"].shape), dw=dw, db=db)
        if s["h0"] is not None:
            out["dh0"] = torch.stack(parts["dh0"])
    return out


def _exact_scan(case, s):
    """Token by token over all sequences side by side (shorter ones stop)."""
    D, N, G = case["D"], case["N"], case["G"]
    A, skip = s["A"].double(), s["D"].double()
    step, train = case["kind"] == "step", case["kind"] == "train"
    rep = D // G
    if step:
        u, z = s["u"].double(), s["z"]
        at = s["slots"].long()
        h = s["h0"].double()
        dt = torch.log(1 + torch.exp(s["delta"].double() + s["bias"].double()))
        Bw = s["B"].double().repeat_interleave(rep, 1)
        Cw = s["C"].double().repeat_interleave(rep, 1)
        hn = torch.exp(dt.unsqueeze(-1) * A) * h[at] + (dt * u).unsqueeze(-1) * Bw
        h[at] = hn
        y = (hn * Cw).sum(-1) + skip * u
        return {"y": y if z is None else y * z.double() / (1 + torch.exp(-z.double())), "state": h}
    spans = _spans(case)
    order = sorted(range(len(spans)), key=lambda i: spans[i][0] - spans[i][1])
    lens = [spans[i][1] - spans[i][0] for i in order]
    start = torch.tensor([spans[i][0] for i in order], device=s["u"].device)

    def rows(x):
        return x.reshape((-1,) + x.shape[2:])

    u, delta, Bf, Cf = rows(s["u"]), rows(s["delta"]), rows(s["B"]), rows(s["C"])
    z = None if s["z"] is None else rows(s["z"])
    bias = s["bias"].double()
    h = torch.zeros(len(spans), D, N, dtype=torch.float64, device=u.device) if s["h0"] is None \
        else s["h0"].double()[order]
    hs = torch.zeros((len(u), D, N), dtype=torch.float64, device=u.device) if train else None
    h_in = h.clone()
    pre = torch.zeros(len(u), D, dtype=torch.float64, device=u.device)
    for t in range(max(lens)):
        m = sum(n > t for n in lens)
        at = start[:m] + t
        dt = torch.log1p(torch.exp(delta[at].double() + bias))
        ut = u[at].double()
        hn = torch.exp(dt.unsqueeze(-1) * A) * h[:m] + \
            (dt * ut).unsqueeze(-1) * Bf[at].double().repeat_interleave(rep, 1)
        h[:m] = hn
        if train:
            hs[at] = hn
        pre[at] = (hn * Cf[at].double().repeat_interleave(rep, 1)).sum(-1) + skip * ut
    back = torch.empty(len(spans), dtype=torch.long, device=u.device)
    back[torch.tensor(order, device=u.device)] = torch.arange(len(spans), device=u.device)
    shape = s["u"].shape
    zd = None if z is None else z.double()
    gate = None if z is None else zd / (1 + torch.exp(-zd))
    out = {"y": (pre if z is None else pre * gate).reshape(shape), "ht": h[back]}
    if not train:
        return out
    gy = rows(s["dy"]).double()
    if z is not None:
        sg = torch.sigmoid(zd)
        out["dz"] = (gy * pre * (sg + zd * sg * (1 - sg))).reshape(shape)
        gy = gy * gate
    du, dd = torch.zeros_like(gy), torch.zeros_like(gy)
    dB = torch.zeros(len(u), G, N, dtype=torch.float64, device=u.device)
    dC, dA = torch.zeros_like(dB), torch.zeros_like(A)
    carry = torch.zeros_like(h)
    for t in range(max(lens) - 1, -1, -1):
        m = sum(n > t for n in lens)
        at = start[:m] + t
        raw = delta[at].double() + bias
        dt, ut = torch.log1p(torch.exp(raw)), u[at].double()
        Bw = Bf[at].double().repeat_interleave(rep, 1)
        g = carry[:m] + Cf[at].double().repeat_interleave(rep, 1) * gy[at].unsqueeze(-1)
        a = torch.exp(dt.unsqueeze(-1) * A)
        p = g * a * (hs[at - 1] if t else h_in[:m])
        gb = (g * Bw).sum(-1)
        du[at] = dt * gb + skip * gy[at]
        dd[at] = ((p * A).sum(-1) + ut * gb) * torch.sigmoid(raw)
        dA += (p * dt.unsqueeze(-1)).sum(0)
        dB[at] = (g * (dt * ut).unsqueeze(-1)).reshape(m, G, rep, N).sum(2)
        dC[at] = (hs[at] * gy[at].unsqueeze(-1)).reshape(m, G, rep, N).sum(2)
        carry[:m] = a * g
    out.update(du=du.reshape(shape), ddelta=dd.reshape(shape), dA=dA, dB=dB.reshape(s["B"].shape),
               dC=dC.reshape(s["C"].shape), dD=(gy * u.double()).sum(0), dbias=dd.sum(0))
    if s["h0"] is not None:
        out["dh0"] = carry[back]
    return out


def _exact_norm(case, s):
    x, G = s["x"].double(), case["G"]
    xg = x.reshape(x.shape[:-1] + (G, -1))
    var, mean = torch.var_mean(xg, -1, correction=0, keepdim=True)
    sd = torch.sqrt(var + 1e-5)
    xh = ((xg - mean) / sd).reshape(x.shape)
    n = xh * s["w"].double() + s["b"].double()
    z = n if s["z"] is None else s["z"].double()
    e = 1 + torch.exp(-z)
    act = z / e
    out = {"y": act if s["z"] is None else n * act}
    if case["kind"] == "train":
        dy = s["dy"].double()
        slope = (1 + z * (1 - 1 / e)) / e
        dn = dy * (slope if s["z"] is None else act)
        if s["z"] is not None:
            out["dz"] = dy * n * slope
        g = (dn * s["w"].double()).reshape(xg.shape)
        xr = xh.reshape(xg.shape)
        m = xg.shape[-1]
        out["dx"] = ((g - g.sum(-1, keepdim=True) / m - xr * (g * xr).sum(-1, keepdim=True) / m)
                     / sd).reshape(x.shape)
        out["dw"] = (dn * xh).flatten(0, 1).sum(0)
        out["db"] = dn.flatten(0, 1).sum(0)
    return out


def exact(case, seed):
    lens = _lens(case) or [case["T"]]
    if case["op"] == "scan" and case["kind"] == "train" and \
            case["B"] * case["T"] * case["D"] * case["N"] * 8 > 80e9:
        return None  # the states in 64 bits would not fit beside the rest
    if case["op"] == "scan" and max(lens) > 20000:
        return None
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm}[case["op"]](case, s)
