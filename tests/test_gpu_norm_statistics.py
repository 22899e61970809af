"""Statistics of rows whose values are nothing like independent: outliers exactly in the channels that the kernels sample for their
pivot (one of every d / 32 of a CTA's columns), and rows far from zero, at one level or at several.  Float32 streams and branches, so
that no output rounding hides what a statistic loses.  Definitions and tolerances are those of test_gpu_norm: a statistic is off
by at most 40 roundings of 2^-24, every value by at most 64 * 2^-24 (gradients 128 * 2^-24) of the terms that make it up."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests.test_gpu_norm import _case, _check, _check_gradients, _forward, _gen, _gradients, _rand

pytestmark = pytest.mark.gpu


def sampled_channels(d, backward):
    """Channels that lie at a sampled place: of the whole row, or of each CTA's columns in the backward pass (clusters of 1, 2, 4)."""
    cluster, groups = 1, (d + 7) // 8
    while backward and groups > 576 * cluster:
        cluster *= 2
    columns = (groups + cluster - 1) // cluster * 8
    return [c0 + lane * min(columns, d - c0) // 32 for c0 in range(0, d, columns) for lane in range(32)]


def shaped(v, kind, backward):
    """What the rows of a test look like."""
    d = v.shape[1]
    idx = torch.tensor(sampled_channels(d, backward), device="cuda")
    if kind == "outliers":
        v[:, idx] += 300.0
    elif kind == "loud outliers":
        v[:, idx] *= 1000.0
        v[:, idx] += 4000.0
    elif kind == "every other row":
        v[1::2, idx] -= 500.0
    elif kind == "far from zero":
        v += 1000.0
    else:                                                    # levels: the first columns, the middle and the last at their own
        v[:, : d // 3] += 100.0
        v[:, -(d // 5):] -= 60.0
    return v


KINDS = ["outliers", "loud outliers", "every other row", "far from zero", "levels"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,branch", [(1032, torch.float32), (2240, torch.float32), (4096, torch.float32), (8192, torch.float32), (16384, torch.bfloat16)])
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("layer", "layer"), ("rms", "layer")])
def test_forward(kind, d, branch, norm, post):
    for rows in (5, 597):                                    # a CTA per row; persistent CTAs
        x, y, s = _case(rows, d, torch.float32, branch, d, norm=norm, post=post)
        shaped(x, kind, False)
        shaped(y, kind, False)
        h, n = kb.kroquant_norm_residual(x, y, **s)
        ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, rows)
        _check(h, ref_h, tol_h)
        _check(n, ref_n, tol_n)
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [1032, 2240, 8192])
def test_forward_without_branch(kind, d):
    x, _, s = _case(600, d, torch.float32, torch.float32, d + 1, gated=False)
    shaped(x, kind, False)
    h, n = kb.kroquant_norm_residual(x, **s)
    ref_h, tol_h, ref_n, tol_n = _forward(x, None, s, 600)
    _check(h, ref_h, tol_h)
    _check(n, ref_n, tol_n)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [200, 512, 640, 1153, 2240, 4608, 4616, 8192, 9001, 12288, 16384])
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("layer", "layer"), ("rms", "layer"), ("none", "layer")])
def test_backward(kind, d, norm, post):
    for rows in (3, 317):
        x, y, s = _case(rows, d, torch.float32, torch.float32, d + rows, norm=norm, post=post)
        shaped(x, kind, True)
        shaped(y, kind, True)
        g = _gen(1)
        dn = _rand(g, torch.float32, rows, d) if norm != "none" else None
        dh = _rand(g, torch.float32, rows, d)
        got = kb.kroquant_norm_residual_grad(dn, x, dh=dh, y=y, **s)
        _check_gradients(got, *_gradients(dn, dh, x, y, s, rows), rows, s)
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("d", [2240, 12288])
def test_the_same_rows_alone_and_among_others(d):
    """A row's statistics are as good in a large call as in a small one."""
    x, y, s = _case(600, d, torch.float32, torch.float32 if d < 8193 else torch.bfloat16, 7, post="layer")
    shaped(x, "outliers", False)
    h, n = kb.kroquant_norm_residual(x, y, **s)
    h1, n1 = kb.kroquant_norm_residual(x[:4].contiguous(), y[:4].contiguous(), **s)
    _, tol_h, _, tol_n = _forward(x[:4], y[:4], s, 4)
    _check(h[:4], h1.double(), 2 * tol_h)
    _check(n[:4], n1.double(), 2 * tol_n)
