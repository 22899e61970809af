"""kroquant_linear_mxfp4_grouped with offsets that are not sorted: a group begins no earlier than the groups before it
end, so that the work stays within what the host allowed for, and rows of no group keep what they held.

Tolerance: that of the sorted groups (float32 output: accumulation of exact products within 1e-6 sum|a||b|, and 2^-23 of the value)."""
import math

import numpy as np
import pytest
import torch

from oracle import c_oracle as co
from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu


def _quantized(rows, K, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.randn(rows, K, device="cuda", generator=g) / math.sqrt(K) * 4).to(torch.bfloat16)
    q, s = kb.kroquant_mxfp4_quantize(x, scale_layout="tiled")
    qr, sr = kb.kroquant_mxfp4_quantize(x)
    return q, s, torch.from_numpy(co.dequantize(qr.cpu().numpy(), sr.cpu().numpy()).astype(np.float64)).cuda()


def owners(offsets, M):
    """Expert of every row, -1: none."""
    owner, end = np.full(M, -1), 0
    for e in range(len(offsets) - 1):
        lo, hi = max(offsets[e], 0), min(offsets[e + 1], M)
        if hi > lo:
            owner[max(lo, end):hi] = e
            end = max(end, hi)
    return owner


def sawtooth(E, M):
    return [0 if e % 2 == 0 else M for e in range(E + 1)]


CASES = [(400, sawtooth(10, 400)),                        # every other group holds all rows
         (20, sawtooth(40, 20)), (1, sawtooth(9, 1)), (64, sawtooth(5, 64)),
         (400, [400, 0, 400, 0, 400, 0]),
         (400, [0, 300, 100, 350, 20, 400, 390]),         # overlaps that reach further each time
         (130, [500, -3, 70, 10, 60, 130, 0, 10 ** 9]),
         (1500, [0, 900, 300, 1200, 1100, 1500]),         # enough rows per weight for the kernel on CTA pairs
         (1500, sawtooth(4, 1500)),
         (2000, list(range(2000, 1960, -1)) + [2000])]    # 39 empty groups and a late one


@pytest.mark.parametrize("M,offsets", CASES, ids=[f"{M}-{i}" for i, (M, _) in enumerate(CASES)])
@pytest.mark.parametrize("N,K", [(96, 1152), (700, 2240)])
def test_decreasing_offsets(M, offsets, N, K):
    E = len(offsets) - 1
    qa, sa, a = _quantized(M, K, 1)
    w = [_quantized(N, K, 10 + e) for e in range(min(E, 4))]
    qw, sw = (torch.stack([w[e % 4][i] for e in range(E)]) for i in range(2))
    owner = torch.from_numpy(owners(offsets, M)).cuda()
    for _ in range(2):
        out = torch.full((M, N), 77.0, device="cuda")
        kb.kroquant_linear_mxfp4_grouped(qa, sa, qw, sw, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out)
        torch.cuda.synchronize()
        assert kb.kroquant_last_device_error() == 0
        assert bool((out[owner < 0] == 77).all())
        for e in range(E):
            rows = owner == e
            if bool(rows.any()):
                ref, size = a[rows] @ w[e % 4][2].t(), a[rows].abs() @ w[e % 4][2].abs().t()
                assert bool(((out[rows].double() - ref).abs() <= 1e-6 * size + 2.0 ** -23 * ref.abs()).all())
