"""Blocks of a recurrent model from the library's operators: trained, prompted and
continued token by token.

    r, n       = stream and first block's input        comba_block_norm, of the embeddings
    q, k, v, f = in_proj(n);  g = log sigmoid(f + b)   torch product
    o          = decay attention(q, k, v, g)           comba_decay, with its state
    y, z       = out_proj(o)                           torch product
    r, n       = r + s norm(y) silu(z), norm(r)        comba_block_norm: into the next block

q, k, v and f, y and z go in as the column slices that the projections leave; pairs of
heads share their keys and values; the stream r stays in fp32.  Run it:

    python examples/decay_blocks.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_02475_amd as comba  # noqa: E402


class DecayBlock(torch.nn.Module):
    def __init__(self, model, heads, dk, dv, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.shared, self.dk, self.dv = heads, max(1, heads // 2), dk, dv
        f = dict(device=device, dtype=torch.float32)
        self.parts = [heads * dk, self.shared * dk, self.shared * dv, heads]
        self.in_proj = torch.nn.Linear(model, sum(self.parts), bias=False, device=device,
                                       dtype=dtype)
        self.out_proj = torch.nn.Linear(heads * dv, 2 * model, bias=False, device=device,
                                        dtype=dtype)
        # time constants of about 5 to 500 tokens
        self.gate_bias = torch.nn.Parameter(torch.linspace(1.5, 6.0, heads, **f))
        self.post_norm = torch.nn.Parameter(torch.ones(model, **f))
        self.scale = torch.nn.Parameter(torch.full((model,), 0.5, **f))
        self.next_norm = torch.nn.Parameter(torch.ones(model, **f))

    def split(self, n):
        """q, k, v of each head (column slices), and the log-decays."""
        q, k, v, f = self.in_proj(n).split(self.parts, -1)
        g = torch.nn.functional.logsigmoid(f.float() + self.gate_bias)
        return (q.unflatten(-1, (self.heads, self.dk)), k.unflatten(-1, (self.shared, self.dk)),
                v.unflatten(-1, (self.shared, self.dv)), g)

    def join(self, o):
        """The block's output and its gate, as slices of one projection."""
        return self.out_proj(o.flatten(-2)).chunk(2, -1)


class DecayBlocks(torch.nn.Module):
    def __init__(self, model=512, layers=2, heads=8, dk=64, dv=64, device="cuda"):
        super().__init__()
        self.first_norm = torch.nn.Parameter(torch.ones(model, device=device))
        self.blocks = torch.nn.ModuleList(DecayBlock(model, heads, dk, dv, device)
                                          for _ in range(layers))

    def forward(self, h, states=None, **packed):
        """h [B,T,model]: (out, every block's state); ``states`` continues earlier tokens,
        ``packed``: cu_seqlens (and cu_seqlens_host) of a packed batch."""
        r, n = comba.comba_block_norm(h, None, self.first_norm, stream_dtype=torch.float32)
        after = []
        for i, b in enumerate(self.blocks):
            o, state = comba.comba_decay(*b.split(n), None if states is None else states[i],
                                         **packed)
            y, z = b.join(o)
            r, n = comba.comba_block_norm(y, r, b.next_norm, post_weight=b.post_norm, z=z,
                                          scale=b.scale)
            after.append(state)
        return n, after

    @torch.no_grad()
    def step(self, h, pools, slots):
        """One token per row, h [B,model]; ``pools`` (a block's states [S,H,dk,dv]) are updated
        in place at each row's slot."""
        r, n = comba.comba_block_norm_fwd(h, None, self.first_norm, stream_dtype=torch.float32)
        for b, pool in zip(self.blocks, pools):
            y, z = b.join(comba.comba_decay_step(*b.split(n), pool, slots=slots))
            r, n = comba.comba_block_norm_fwd(y, r, b.next_norm, post_weight=b.post_norm, z=z,
                                              scale=b.scale)
        return n


def train(model, steps=20, B=4, T=256):
    """Fits a fixed random target; returns the losses."""
    width = model.first_norm.numel()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    h = torch.randn(B, T, width, device="cuda", generator=gen).bfloat16()
    target = torch.randn(B, T, width, device="cuda", generator=gen)
    opt = torch.optim.Adam(model.parameters(), lr=1e-3)
    losses = []
    for _ in range(steps):
        out, _ = model(h)
        loss = (out.float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def serve(model, lens=(70, 1, 133), new=5):
    """Prompts of unequal length packed into one call, their states placed in pools, then
    ``new`` tokens per request one at a time.  Returns (stepped outputs, the same tokens from
    one packed call over everything), [requests, new, model] each."""
    width = model.first_norm.numel()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    hs = [torch.randn(n + new, width, device="cuda", generator=gen).bfloat16() for n in lens]

    def packed(parts):
        cu = torch.tensor([0] + [len(p) for p in parts], dtype=torch.int32).cumsum(0).int()
        kw = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu.numpy())
        return torch.cat(parts)[None], kw, cu.tolist()

    x, kw, _ = packed([h[:n] for h, n in zip(hs, lens)])
    _, states = model(x, **kw)
    slots = torch.arange(len(lens), device="cuda", dtype=torch.int32) * 2 + 1  # anywhere
    pools = [s.new_zeros((2 * len(lens) + 1,) + s.shape[1:]) for s in states]
    for p, s in zip(pools, states):
        p[slots.long()] = s
    got = [model.step(torch.stack([h[n + k] for h, n in zip(hs, lens)]), pools, slots)
           for k in range(new)]
    x, kw, cu = packed(hs)
    whole, _ = model(x, **kw)
    want = torch.stack([whole[0, b - new:b] for b in cu[1:]])
    return torch.stack(got, 1), want


if __name__ == "__main__":
    torch.manual_seed(0)
    blocks = DecayBlocks()
    losses = train(blocks)
    print("loss %.4f -> %.4f" % (losses[0], losses[-1]))
    got, want = serve(blocks)
    print("steps against one call: largest difference %.2e of %.2e"
          % ((got - want).float().abs().max().item(), want.float().abs().max().item()))
