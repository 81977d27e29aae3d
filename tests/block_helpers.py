"""Shared by the tests of a block's operators: inputs on the device, cases, bounds."""
import numpy as np

from comba_inputs import bf16_round


def dt(name):
    import torch

    return torch.bfloat16 if name == "bf16" else torch.float32


def dev(x, dtype=None):
    import torch

    return None if x is None else \
        torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype or torch.float32)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def column_slice(x, dtype, lead, before=0, after=0):
    """x on the device as a column slice of wider rows (``lead`` leading dimensions of tokens);
    the rows' other columns hold NaN."""
    import torch

    if x is None:
        return None
    n = int(np.prod(x.shape[lead:]))
    wide = torch.full(x.shape[:lead] + (before + n + after,), float("nan"), device="cuda",
                      dtype=dtype)
    wide[..., before:before + n] = dev(x, dtype).reshape(x.shape[:lead] + (n,))
    return wide[..., before:before + n].unflatten(-1, x.shape[lead:])


def rnd(rng, dtype, *shape, scale=1.0):
    x = (scale * rng.standard_normal(shape)).astype(np.float32)
    return bf16_round(x) if dtype == "bf16" else x


def spans(B, T, lens):
    ends = np.cumsum([0] + list([T] * B if lens is None else lens))
    return [(int(a), int(b)) for a, b in zip(ends[:-1], ends[1:])]


def packed(lens, with_host):
    import torch

    if lens is None:
        return {}
    cu = np.cumsum([0] + list(lens)).astype(np.int32)
    kw = {"cu_seqlens": dev(cu, torch.int32)}
    if with_host:
        kw["cu_seqlens_host"] = cu
    return kw


HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step of a rounding, relative


def hold(name, got, want, magnitude, dtype, inner=1):
    """fp32: a norm-wise max relative error of 1e-5 (the repository's bar: sums of up to some
    1e4 terms of 2^-24 each).  bf16: the output's own rounding, half a step of the value; each
    term of its sum has ``inner`` factors rounded to bf16 (pair weights or states), so as many
    half steps of the sum of the terms' absolute values, ``magnitude`` (the same formula on
    absolute inputs); the fp32 sums' 1e-5 of it.  Those are the worst cases; roundings are
    independent, an rms of 0.42 half steps each (a mantissa uniform in its logarithm), so that the
    tensor's 2-norm is held to sqrt(inner + 1) times that, and half of it more."""
    got = host(got).reshape(np.shape(want))
    if want.size == 0:
        return
    assert np.all(np.isfinite(got)), name
    err = np.abs(got - want)
    if dtype == "f32":
        worst = np.max(err) / max(np.max(np.abs(want)), 1e-30)
        assert worst <= 1e-5, (name, worst)
        return
    h = HALF[dtype]
    over = err - (h * (1 + h) ** inner * np.abs(want) + (inner * h * (1 + h) ** inner + 1e-5) * magnitude)
    assert np.max(over) <= 0, (name, np.max(over), np.max(err))
    if want.size >= 1000:
        rel = np.linalg.norm(got - want) / np.linalg.norm(want)
        assert rel <= 1.5 * 0.42 * h * np.sqrt(inner + 1), (name, rel)
