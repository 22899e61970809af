"""A quantized feed-forward block and its mixture-of-experts form on the library's own kernels, and the backward pass of the
step between the blocks:

    h, n = norm_residual(x, attention branch)        adaptive norm, gated residual         one launch
    u    = silu(Q(n) Wg^T + b) * (Q(n) Wv^T + b)     quantizer + gated W4A4 product        two launches
    x'   = h + gate * (Q(u) Wo^T)                    quantizer + W4A4 product, residual    two launches

    python examples/quantized_block.py [--tokens 4096] [--width 2240] [--hidden 5600] [--experts 8]

Synthetic weights and activations; the outputs are compared with the same block in float32 without quantization."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_21446_b200 import binding as kb  # noqa: E402
from paper_2607_21446_b200 import workloads as wl  # noqa: E402


def randn(g, *shape, gain=1.0, dtype=torch.bfloat16):
    return (gain * torch.randn(*shape, device="cuda", generator=g)).to(dtype)


def dense_layer(W):
    """W4A4 layer with the Hadamard initialisation of the Kronecker factors (what calibration starts from) on the activations and
    its inverse transpose on the weights."""
    import numpy as np
    a, b, c = (wl.hadamard_lu_params()[0, :, i].astype(np.float64) for i in range(3))
    G = np.stack([[[[a[k], b[k]], [a[k] * c[k], b[k] * c[k] - 1 / a[k]]] for k in range(5)]])
    H = np.stack([[np.linalg.inv(G[0, k]).T for k in range(5)]])
    return kb.LinearW4A4.from_weights(W, G.astype(np.float32), H.astype(np.float32))


def run(tokens=4096, width=2240, hidden=5600, experts=8, batches=2, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x, branch = randn(g, tokens, width), randn(g, tokens, width)
    gate, scale, shift, gate_out = (randn(g, batches, width, gain=0.3, dtype=torch.float32) for _ in range(4))
    Wg, Wv = randn(g, hidden, width, gain=width ** -0.5), randn(g, hidden, width, gain=width ** -0.5)
    Wo = randn(g, width, hidden, gain=hidden ** -0.5)

    # ---- the block ----
    h, n = kb.kroquant_norm_residual(x, branch, gate=gate, scale=scale, shift=shift, norm="layer")
    first, second = dense_layer(kb.interleave_glu(Wg, Wv)), dense_layer(Wo)
    u = first.fused(n, features=hidden, activation="silu", glu=True)
    y = second.fused(u, gate=gate_out, residual=h)

    per = tokens // batches
    wide = lambda v: v.repeat_interleave(per, 0)  # noqa: E731
    h32 = x.float() + wide(gate) * branch.float()
    n32 = torch.nn.functional.layer_norm(h32, (width,), eps=1e-6) * (1 + wide(scale)) + wide(shift)
    u32 = torch.nn.functional.silu(n32 @ Wg.float().t()) * (n32 @ Wv.float().t())
    y32 = h32 + wide(gate_out) * (u32 @ Wo.float().t())
    error = float((y.float() - y32).norm() / (y32 - h32).norm())

    # ---- the same with experts: rows sorted by expert, offsets on the device, nothing padded ----
    choice = torch.randint(0, experts, (tokens,), device="cuda", generator=g)
    order = torch.argsort(choice, stable=True)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.bincount(choice, minlength=experts).cumsum(0)
    weight = torch.rand(tokens, device="cuda", generator=g)
    stacks = []
    for rows, cols in ((2 * hidden, width), (width, hidden)):
        parts = [kb.kroquant_mxfp4_quantize(randn(g, rows, cols, gain=cols ** -0.5), scale_layout="tiled") for _ in range(experts)]
        stacks.append((torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])))
    (w1, s1), (w2, s2) = stacks
    q, s = kb.kroquant_mxfp4_quantize(n[order].contiguous(), scale_layout="tiled")
    glu_hidden = w1.shape[1] // 2 // 32 * 32
    u_e = kb.kroquant_linear_mxfp4_grouped(q, s, w1, s1, offsets, features=glu_hidden, activation="silu", glu=True)
    q, s = kb.kroquant_mxfp4_quantize(u_e, scale_layout="tiled")
    moe = kb.kroquant_linear_mxfp4_grouped(q, s, w2, s2, offsets, row_scale=weight[order].contiguous(), residual=h[order].contiguous())

    # ---- gradients of the step between the blocks ----
    grads = kb.kroquant_norm_residual_grad(torch.ones_like(n), h, dh=torch.ones_like(h), y=branch, gate=gate, scale=scale, shift=shift, norm="layer")
    torch.cuda.synchronize()
    assert kb.kroquant_last_device_error() == 0
    return {"relative_error": error, "out": y, "moe": moe, "grads": grads}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4096), ("width", 2240), ("hidden", 5600), ("experts", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    r = run(a.tokens, a.width, a.hidden, a.experts)
    print(f"block: relative error of the branch against float32 {r['relative_error']:.3f} (4-bit weights and activations); "
          f"experts: {tuple(r['moe'].shape)}; gradients: {sorted(r['grads'])}")
