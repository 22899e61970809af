"""Forms of the linear layer's epilogue in combination: the gated product with gate, row scale and residual, groups with a residual, and
operands of different types in one call.  Definitions and tolerances are those of test_gpu_linear."""
import itertools

import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests.test_gpu_linear import _check, _check_device, _gen, _groups, _quantized, _reference

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _rand(g, dt, *shape):
    return torch.randn(*shape, device="cuda", generator=g).to(dt)


def _rows(N, glu):
    return 64 * ((N + 31) // 32) if glu else N


@pytest.mark.parametrize("M,N", [(7, 64), (48, 101), (96, 320), (300, 200), (774, 577), (1500, 1024)])
@pytest.mark.parametrize("res,out", [(BF16, BF16), (F32, BF16), (F16, F32), (F32, F32), (BF16, F16)])
def test_gated_product_with_gate_row_scale_and_residual(M, N, res, out):
    """16 features a chunk: whole, half-filled and ragged copies of the residual; one gate row, several, and one per row."""
    K, R, g = 544, _rows(N, True), _gen(M + N)
    qa, sa, a = _quantized(M, K, 1)
    qw, sw, w = _quantized(R, K, 2)
    bias, residual, row_scale = _rand(g, F32, R), _rand(g, res, M, N), torch.rand(M, device="cuda", generator=g)
    for batches, per in ((0, None), (1, None), (3, (M + 2) // 3), (M, 1)):
        gate = _rand(g, F32, batches, N) if batches else None
        o = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, features=N, bias=bias, activation="silu", glu=True, gate=gate, rows_per_gate=per,
                                     row_scale=row_scale, residual=residual, residual_scale=0.5, out_dtype=out)
        full = None if gate is None else gate.repeat_interleave(per or M, 0)[:M]
        _check(o, *_reference(a, w, N, "silu", True, bias, full, row_scale, residual, 0.5))
    _check_device()


@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("M,N", [(9, 96), (400, 200)])
@pytest.mark.parametrize("res,gate,bias,out", list(itertools.product((F32, BF16), (F16, F32), (BF16, F32), (F16, F32)))[::2] + [(F16, BF16, F16, BF16)])
def test_operands_of_different_types(M, N, glu, res, gate, bias, out):
    K, R, g = 288, _rows(N, glu), _gen(7)
    qa, sa, a = _quantized(M, K, 3)
    qw, sw, w = _quantized(R, K, 4)
    b, y, r = _rand(g, bias, R), _rand(g, gate, 2, N), _rand(g, res, M, N)
    per = (M + 1) // 2
    o = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, features=N, bias=b, activation="relu", glu=glu, gate=y, rows_per_gate=per, residual=r, out_dtype=out)
    _check(o, *_reference(a, w, N, "relu", glu, b, y.repeat_interleave(per, 0)[:M], None, r))
    _check_device()


@pytest.mark.parametrize("M", [11, 500])
@pytest.mark.parametrize("shift,pitch", [(0, 0), (1, 7), (8, 8), (16, 40)])
@pytest.mark.parametrize("N", [200, 72])
def test_gated_product_in_place_at_odd_places(M, shift, pitch, N):
    """out is the residual itself, with canaries around every row."""
    K, R = 288, _rows(N, True)
    qa, sa, a = _quantized(M, K, 5)
    qw, sw, w = _quantized(R, K, 6)
    flat = torch.full((shift + M * (N + pitch),), 77.0, dtype=BF16, device="cuda")
    view = flat[shift:].view(M, N + pitch)[:, :N]
    res = _rand(_gen(8), BF16, M, N)
    view.copy_(res)
    kb.kroquant_linear_mxfp4(qa, sa, qw, sw, features=N, glu=True, activation="silu", residual=view, out=view)
    _check(view, *_reference(a, w, N, "silu", True, residual=res))
    assert bool((flat[:shift] == 77).all()) and bool((flat[shift:].view(M, N + pitch)[:, N:] == 77).all())
    _check_device()


@pytest.mark.parametrize("sizes", [[5, 0, 3, 8], [100] * 7, [700, 0, 3, 513], [2000, 1]], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("res,out", [(BF16, BF16), (F32, F16), (F16, F32)])
@pytest.mark.parametrize("N", [160, 161])
def test_groups_with_a_residual(sizes, glu, res, out, N):
    """Groups that share row tiles: every row takes its own residual, rows outside the groups keep theirs (out is not written there)."""
    T, E, K, R, g = sum(sizes) + 6, len(sizes), 544, _rows(N, glu), _gen(9)
    qa, sa, a = _quantized(T, K, 10)
    w = [_quantized(R, K, 20 + e) for e in range(E)]
    residual, row_scale = _rand(g, res, T, N), torch.rand(T, device="cuda", generator=g)
    offsets = _groups(sizes) + 4
    o = torch.full((T, N), 77.0, device="cuda", dtype=out)
    kb.kroquant_linear_mxfp4_grouped(qa, sa, torch.stack([x[0] for x in w]), torch.stack([x[1] for x in w]), offsets, features=N,
                                     activation="gelu", glu=glu, row_scale=row_scale, residual=residual, residual_scale=2.0, out=o)
    lo = 4
    for e, n in enumerate(sizes):
        if n:
            rows = slice(lo, lo + n)
            _check(o[rows], *_reference(a[rows], w[e][2], N, "gelu", glu, None, None, row_scale[rows], residual[rows], 2.0))
        lo += n
    assert bool((o[:4] == 77).all()) and bool((o[lo:] == 77).all())
    _check_device()
