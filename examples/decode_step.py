"""A transformer block with MXFP4 weights run token by token: a prompt goes through it as one chunk, then every sequence takes one
token at a time on the library's own kernels:

    n        = norm(x)                                                           one launch
    q, k, v  = (n T) Wqkv^T        rows in 16 bits, weights in MXFP4              two launches
    q, k     = rotary(q, k)        time, height and width axes, or one           one launch
    cache   <- k, v                MXFP8, MXFP4 or 16 bits, paged                 one launch
    o        = attention(q, cache)                                                one or two launches
    x        = x + (o T) Wo^T                                                     two launches

    python examples/decode_step.py [--width 1152] [--heads 16] [--kv-heads 4] [--prompt 300] [--steps 8] [--format mxfp8]

Synthetic weights and activations; the outputs are compared with the same block in float32 with unquantized weights and cache."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.quantized_block import dense_layer, randn  # noqa: E402
from paper_2607_21446_b200 import binding as kb  # noqa: E402


class Block:
    """One block's weights, its cache and the pages of its sequences."""

    def __init__(self, width, heads, kv_heads, head_dim, sequences, room, page_size, form, g, axes=None):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.Wqkv = randn(g, (heads + 2 * kv_heads) * head_dim, width, gain=width ** -0.5)
        self.Wo = randn(g, width, heads * head_dim, gain=(heads * head_dim) ** -0.5)
        self.qkv, self.proj = dense_layer(self.Wqkv), dense_layer(self.Wo)
        self.norm = 1 + 0.1 * torch.randn(width, device="cuda", generator=g)
        self.axes = (head_dim,) if axes is None else axes
        self.frequencies = kb.rotary_frequencies(self.axes)
        per = (room + page_size - 1) // page_size
        self.cache = kb.KVCache.empty(sequences * per, page_size, kv_heads, head_dim, form)
        order = torch.randperm(sequences * per, generator=torch.Generator().manual_seed(0))
        self.table = order.view(sequences, per).to(torch.int32).cuda()
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device="cuda")

    def split(self, qkv):
        H, KV = self.heads, self.kv_heads
        q, k, v = qkv.unflatten(1, (H + 2 * KV, self.head_dim)).split((H, KV, KV), 1)
        return q, k, v

    def prompt(self, x, offsets, positions):
        """x [rows, width], packed; fills the cache (the chunk's own attention is not the point here)."""
        _, n = kb.kroquant_norm_residual(x, weight=self.norm)
        q, k, v = self.split(self.qkv.fused(n))
        q, k = kb.kroquant_rotary(q, k, positions, self.frequencies, axes=self.axes, layout="half", out=(q, k))
        kb.kroquant_cache_write(self.cache, k, v, self.table, offsets=offsets)
        self.lengths.copy_(offsets[1:] - offsets[:-1])

    def step(self, x, positions):
        """x [sequences, width], one token of each; positions [sequences, axes]."""
        _, n = kb.kroquant_norm_residual(x, weight=self.norm)
        q, k, v = self.split(self.qkv.few(n))
        q, k = kb.kroquant_rotary(q, k, positions, self.frequencies, axes=self.axes, layout="half", out=(q, k))
        kb.kroquant_cache_write(self.cache, k, v, self.table, starts=self.lengths)
        self.lengths += 1
        o = kb.kroquant_cache_attention(q, self.cache, self.table, self.lengths)
        return self.proj.few(o.flatten(1), residual=x)


def reference_step(block, history, x, positions):
    """The same step in float32 with the weights as they were; history: (keys, values) of every sequence."""
    n = x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6) * block.norm
    q, k, v = block.split(n @ block.Wqkv.float().t())
    q, k = kb.kroquant_rotary(q.contiguous(), k.contiguous(), positions, block.frequencies, axes=block.axes, layout="half")
    rows = []
    for s in range(x.shape[0]):
        keys, values = (torch.cat([h, t[s : s + 1]]) for h, t in zip(history[s], (k, v)))
        history[s] = (keys, values)
        qs = q[s].view(block.kv_heads, -1, block.head_dim)
        w = torch.softmax(block.head_dim ** -0.5 * qs @ keys.permute(1, 2, 0), -1)
        rows.append((w @ values.transpose(0, 1)).reshape(-1))
    return x.float() + torch.stack(rows) @ block.Wo.float().t()


def run(width=1152, heads=16, kv_heads=4, head_dim=72, sequences=3, prompt=300, steps=8, form="mxfp8", page_size=16, axes=None, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    block = Block(width, heads, kv_heads, head_dim, sequences, prompt + steps, page_size, form, g, axes)
    sizes = [max(1, prompt - 37 * i) for i in range(sequences)]
    offsets = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).cuda()
    place = torch.cat([torch.arange(n) for n in sizes]).to(torch.int32).cuda()
    spread = lambda t: torch.stack([t // (i * 3 + 1) for i in range(len(block.axes))], -1).to(torch.int32).contiguous()  # noqa: E731
    x = randn(g, int(offsets[-1]), width)
    block.prompt(x, offsets, spread(place))
    # float32 history from unquantized weights
    n = x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6) * block.norm
    q, k, v = block.split(n @ block.Wqkv.float().t())
    _, k = kb.kroquant_rotary(q.contiguous(), k.contiguous(), spread(place), block.frequencies, axes=block.axes, layout="half")
    at = offsets.tolist()
    history = [(k[a:b], v[a:b]) for a, b in zip(at[:-1], at[1:])]
    errors, token = [], randn(g, sequences, width)
    for _ in range(steps):
        positions = spread(block.lengths.clone())
        want = reference_step(block, history, token, positions)
        out = block.step(token, positions)
        errors.append(float((out.float() - want).norm() / (want - token.float()).norm()))
        token = randn(g, sequences, width)
    keys, values = kb.kroquant_cache_read(block.cache, block.table, int(block.lengths.sum()),
                                          offsets=torch.cat([block.lengths.new_zeros(1), block.lengths.cumsum(0).to(torch.int32)]))
    torch.cuda.synchronize()
    assert kb.kroquant_last_device_error() == 0
    return {"errors": errors, "out": out, "keys": keys, "values": values, "block": block, "history": history}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 1152), ("heads", 16), ("kv-heads", 4), ("head-dim", 72), ("sequences", 3), ("prompt", 300), ("steps", 8), ("page-size", 16)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--format", default="mxfp8", choices=sorted(kb.CACHE_FORMATS))
    a = ap.parse_args()
    r = run(a.width, a.heads, a.kv_heads, a.head_dim, a.sequences, a.prompt, a.steps, a.format, a.page_size)
    print(f"{a.steps} steps of {a.sequences} sequences, cache {a.format}: relative error of the branch against float32 "
          f"{min(r['errors']):.3f} to {max(r['errors']):.3f} (4-bit weights)")
