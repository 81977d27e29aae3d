"""A selective recurrent layer from the library's operators: trained, prompted and
continued token by token.

    x, z   = in_proj(h)                         torch product
    x      = silu(conv(x))                      comba_conv, with its history
    d, B, C = x_proj(x);  delta = dt_proj(d)    torch products
    y      = scan(x, delta, A, B, C, D)         comba_select, with its state
    y      = group_norm(y) * silu(z)            comba_group_norm, gated
    out    = out_proj(y)                        torch product

x, z, B and C go in as the column slices that the projections leave.  Run it:

    python examples/selective_layer.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_02475_amd as comba  # noqa: E402


class SelectiveLayer(torch.nn.Module):
    def __init__(self, model=512, inner=1024, states=16, taps=4, groups=8, device="cuda",
                 dtype=torch.bfloat16):
        super().__init__()
        self.inner, self.states, self.groups = inner, states, groups
        self.rank = rank = inner // 32
        f = dict(device=device, dtype=torch.float32)

        def linear(i, o):
            return torch.nn.Linear(i, o, bias=False, device=device, dtype=dtype)

        self.in_proj, self.out_proj = linear(model, 2 * inner), linear(inner, model)
        self.x_proj, self.dt_proj = linear(inner, rank + 2 * states), linear(rank, inner)
        self.conv_w = torch.nn.Parameter(torch.randn(inner, taps, **f) / math.sqrt(taps))
        self.conv_b = torch.nn.Parameter(torch.zeros(inner, **f))
        self.A_log = torch.nn.Parameter(torch.arange(1, states + 1, **f).log().repeat(inner, 1))
        self.D = torch.nn.Parameter(torch.ones(inner, **f))
        step = torch.exp(torch.rand(inner, **f) * math.log(100) + math.log(0.001))
        self.dt_bias = torch.nn.Parameter(step + torch.log(-torch.expm1(-step)))
        self.norm_w = torch.nn.Parameter(torch.ones(inner, **f))
        self.norm_b = torch.nn.Parameter(torch.zeros(inner, **f))

    def _split(self, x):
        p = self.x_proj(x)
        d, B, C = p.split([self.rank, self.states, self.states], -1)
        return self.dt_proj(d), B, C

    def forward(self, h, states=None, **packed):
        """h [B,T,model]: (out, (conv history, scan state)); ``states`` continues earlier tokens,
        ``packed``: cu_seqlens (and cu_seqlens_host) of a packed batch."""
        conv0, scan0 = states or (None, None)
        x, z = self.in_proj(h).split(self.inner, -1)
        x, conv = comba.comba_conv(x, self.conv_w, self.conv_b, conv0, **packed)
        delta, B, C = self._split(x)
        y, scan = comba.comba_select(x, delta, -self.A_log.exp(), B, C, self.D, None, self.dt_bias,
                                     scan0, **packed)
        y = comba.comba_group_norm(y, self.groups, self.norm_w, self.norm_b, z)
        return self.out_proj(y), (conv, scan)

    @torch.no_grad()
    def step(self, h, pool, slots):
        """One token per row, h [B,model]; ``pool`` (conv histories [S,K-1,inner], scan states
        [S,inner,states]) is updated in place at each row's slot."""
        x, z = self.in_proj(h).split(self.inner, -1)
        x = comba.comba_conv_step(x, self.conv_w, self.conv_b, pool[0], slots=slots)
        delta, B, C = self._split(x)
        y = comba.comba_select_step(x, delta, -self.A_log.exp(), B, C, self.D, None, self.dt_bias,
                                    pool[1], slots=slots)
        y = comba.comba_group_norm_fwd(y, self.groups, self.norm_w, self.norm_b, z)
        return self.out_proj(y)


def train(layer, steps=20, B=4, T=256):
    """Fits a fixed random target; returns the losses."""
    model = layer.in_proj.in_features
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    h = torch.randn(B, T, model, device="cuda", generator=gen).bfloat16()
    target = torch.randn(B, T, model, device="cuda", generator=gen)
    opt = torch.optim.Adam(layer.parameters(), lr=1e-3)
    losses = []
    for _ in range(steps):
        out, _ = layer(h)
        loss = (out.float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def serve(layer, lens=(70, 1, 133), new=5):
    """Prompts of unequal length packed into one call, their states placed in a pool, then
    ``new`` tokens per request one at a time.  Returns (stepped outputs, the same tokens from
    one packed call over everything), [requests, new, model] each."""
    model = layer.in_proj.in_features
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    hs = [torch.randn(n + new, model, device="cuda", generator=gen).bfloat16() for n in lens]

    def packed(parts):
        cu = torch.tensor([0] + [len(p) for p in parts], dtype=torch.int32).cumsum(0).int()
        kw = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu.numpy())
        return torch.cat(parts)[None], kw, cu.tolist()

    x, kw, _ = packed([h[:n] for h, n in zip(hs, lens)])
    _, (conv, scan) = layer(x, **kw)
    slots = torch.arange(len(lens), device="cuda", dtype=torch.int32) * 2 + 1  # anywhere
    pool = tuple(s.new_zeros((2 * len(lens) + 1,) + s.shape[1:]) for s in (conv, scan))
    for p, s in zip(pool, (conv, scan)):
        p[slots.long()] = s
    got = [layer.step(torch.stack([h[n + k] for h, n in zip(hs, lens)]), pool, slots)
           for k in range(new)]
    x, kw, cu = packed(hs)
    whole, _ = layer(x, **kw)
    want = torch.stack([whole[0, b - new:b] for b in cu[1:]])
    return torch.stack(got, 1), want


if __name__ == "__main__":
    torch.manual_seed(0)
    layer = SelectiveLayer()
    losses = train(layer)
    print("loss %.4f -> %.4f" % (losses[0], losses[-1]))
    got, want = serve(layer)
    print("steps against one call: largest difference %.2e of %.2e"
          % ((got - want).float().abs().max().item(), want.float().abs().max().item()))
