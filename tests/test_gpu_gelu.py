"""gelu (erf) of the linear layer on its own: a product of zeros plus a float32 bias hands any value to the activation exactly.

Tolerances, from the arithmetic: for v > 0 the result is v (1 - q), for v < 0 v q, with q = Phi(-|v|) = 2^R and R a polynomial in 32
bits.  The activation is off by at most 2^-23 |v| (error of q: 1.2 * 2^-23 q of the hardware exponential and R's roundings, at most
2^-25 of what q is taken from) and its output rounded once, 2^-23 of the value as for every float32 output here.  R's relative
accuracy falls with its size and the fit's tail: 2^-20 down to -2, 2^-19 to -4, 2^-17 to -6, 2^-14 to -8."""
import math

import pytest
import torch

from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu


def _gelu(values, M, glu=False):
    """gelu of every value, through the kernel that takes M rows."""
    K, R = 64, values.numel()
    qa = torch.zeros(M, K // 2, dtype=torch.uint8, device="cuda")
    sa = torch.full((kb.tiled_scale_bytes(M, K),), 127, dtype=torch.uint8, device="cuda")
    qw = torch.zeros(R, K // 2, dtype=torch.uint8, device="cuda")
    sw = torch.full((kb.tiled_scale_bytes(R, K),), 127, dtype=torch.uint8, device="cuda")
    out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, bias=values, activation="gelu", glu=glu, out_dtype=torch.float32)
    torch.cuda.synchronize()
    assert kb.kroquant_last_device_error() == 0
    assert torch.equal(out[0].expand_as(out).contiguous().view(torch.int32), out.view(torch.int32))
    return out[0].double()


def _exact(v):
    return v.double() * 0.5 * torch.special.erfc(-v.double() / math.sqrt(2))


def _values():
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    u = torch.rand(60000, device="cuda", generator=g)
    return torch.cat([torch.linspace(-8, 8, 40001, device="cuda"), 16 * u[:20000] - 8, torch.exp2(-30 * u[20000:40000]),
                      -torch.exp2(-30 * u[40000:])]).float()


@pytest.mark.parametrize("M", [1, 100])
def test_gelu_is_as_good_as_plain_32_bit_arithmetic(M):
    v = _values()
    ref = _exact(v)
    over = (_gelu(v, M) - ref).abs() - 2.0 ** -23 * (v.double().abs() + ref.abs())
    assert float((over / v.double().abs().clamp_min(1e-30)).max()) <= 0


@pytest.mark.parametrize("M", [1, 100])
@pytest.mark.parametrize("lo,bits", [(-2, 20), (-4, 19), (-6, 17), (-7.99, 14)])
def test_the_negative_tail_keeps_its_digits(M, lo, bits):
    v = torch.linspace(lo, lo / 2, 20001, device="cuda")
    ref = _exact(v)
    assert float(((_gelu(v, M) - ref).abs() / ref.abs()).max()) <= 2.0 ** -bits


@pytest.mark.parametrize("M", [1, 100])
def test_gelu_far_out(M):
    inf, nan = float("inf"), float("nan")
    v = torch.tensor([8.0, 8.5, 30, 1e5, 3e38, inf, -8.0, -8.5, -30, -1e5, -3e38, 0.0, -0.0, 1e-40, nan], device="cuda")
    got = _gelu(torch.cat([v, torch.zeros(17, device="cuda")]), M)
    assert torch.equal(got[:6], v[:6].double())
    assert bool((got[6:13].abs() <= 5e-15).all()) and float(got[13]) >= 0 and bool(torch.isnan(got[14]))


@pytest.mark.parametrize("M", [1, 100])
def test_gated_gelu(M):
    """act(gate half) times a value half of ones."""
    v = torch.linspace(-8, 8, 32 * 64, device="cuda")
    bias = torch.stack([v.view(-1, 32), torch.ones(64, 32, device="cuda")], 1).reshape(-1)
    ref = _exact(v)
    assert bool(((_gelu(bias, M, glu=True) - ref).abs() <= 2.0 ** -23 * (v.double().abs() + ref.abs())).all())
