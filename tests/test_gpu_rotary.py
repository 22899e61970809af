"""Rotary positions against complex numbers in 64 bits.  Per value: one rounding to the type (half a step, finfo.eps / 2 of the value) and
32-bit arithmetic: sine and cosine are within 2^-23 (sincospif 1 unit, its correction and rounding another half), each product and
the sum round once, in all at most 4 * 2^-24 (|a| + |b|)."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def pairs_of(axes, layout):
    n = sum(axes) // 2
    p = torch.arange(n, device="cuda")
    return (2 * p, 2 * p + 1) if layout == "interleaved" else (p, p + n)


def reference(x, positions, freqs, axes, layout, inverse=False):
    """-> value, and |a| + |b| of the pair it comes from (0 where it is copied), float64; x [.., tokens, heads, d]."""
    column = [i for i, a in enumerate(axes) for _ in range(a // 2)]
    angle = positions.double()[..., column] * freqs
    turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle).unsqueeze(-2)
    a, b = pairs_of(axes, layout)
    y, size = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    z = torch.complex(y[..., a], y[..., b])
    size[..., a] = size[..., b] = z.real.abs() + z.imag.abs()
    z = z * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y, size


def check(got, x, positions, freqs, axes, layout, inverse=False):
    want, size = reference(x, positions, freqs, axes, layout, inverse)
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() + 4 * 2.0 ** -24 * size * (1 + torch.finfo(got.dtype).eps)
    tol += torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps           # half a step among the subnormal
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), float(((got.double() - want).abs() - tol).max())
    n = sum(axes)
    assert torch.equal(got[..., n:], x[..., n:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("tokens,heads,kv,d,axes", [
    (1, 32, 8, 128, (128,)), (1, 1, 1, 2, (2,)), (3, 2, 1, 128, (16, 56, 56)), (131, 16, 16, 72, (24, 24, 24)), (1000, 4, 2, 112, (16, 32, 32, 32)),
    (77, 5, 3, 80, (20, 20)), (50, 2, 2, 71, (22, 20)), (9, 3, 1, 256, (64, 2, 62)), (5, 2, 7, 66, (6, 0, 60)), (2, 1, 1, 511, (510,)), (4, 1, 2, 512, (2,)),
    (700, 1, 1, 64, (64,)), (2000, 36, 4, 128, (128,))])
def test_forward_and_backward(dtype, layout, tokens, heads, kv, d, axes):
    g = gen(tokens + d)
    q, k = (torch.randn(tokens, h, d, device="cuda", generator=g).to(dtype) for h in (heads, kv))
    pos = torch.randint(-1000, 100000, (tokens, len(axes)), device="cuda", generator=g, dtype=torch.int32)
    f = kb.rotary_frequencies(axes)
    for inverse in (False, True):
        a, b = kb.kroquant_rotary(q, k, pos, f, axes=axes, layout=layout, inverse=inverse)
        check(a, q, pos, f, axes, layout, inverse)
        check(b, k, pos, f, axes, layout, inverse)
    only = kb.kroquant_rotary(q, None, pos, f, axes=axes, layout=layout)
    check(only, q, pos, f, axes, layout)


@pytest.mark.parametrize("positions", [[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, 2 ** 24 + 1]])
def test_far_positions_keep_their_angle(positions):
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    x = torch.randn(len(positions), 2, 64, device="cuda", generator=gen(0))
    f = kb.rotary_frequencies((64,))
    y = kb.kroquant_rotary(x, None, pos, f)
    # the reference's own angle is rounded to 64 bits: 2^31 * 2^-53 = 2.4e-7 on top of the derived tolerance
    want, size = reference(x, pos[:, None], f, (64,), "interleaved")
    assert bool(((y.double() - want).abs() <= 2.0 ** -24 * want.abs() + (4 * 2.0 ** -24 + 2 * 2.0 ** -22) * size).all())


def test_fractional_positions():
    pos = torch.randn(40, 2, device="cuda", generator=gen(1)) * 300
    x = torch.randn(40, 3, 96, device="cuda", generator=gen(2)).half()
    f = kb.rotary_frequencies((48, 48), theta=100.0)
    check(kb.kroquant_rotary(x, None, pos, f, axes=(48, 48), layout="half"), x, pos, f, (48, 48), "half")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_strides_and_in_place(dtype, layout):
    T, H, KV, d, axes = 37, 6, 2, 64, (32, 16)
    g = gen(3)
    pos = torch.randint(0, 5000, (T, 2), device="cuda", generator=g, dtype=torch.int32)
    f = kb.rotary_frequencies(axes)
    qkv = torch.randn(T, (H + 2 * KV) * d + 3, device="cuda", generator=g).to(dtype)
    before = qkv.clone()

    def views(t):
        return t[:, : H * d].unflatten(1, (H, d)), t[:, H * d : (H + KV) * d].unflatten(1, (KV, d))

    q, k = views(qkv)                                                    # an odd row pitch: single elements
    a, b = kb.kroquant_rotary(q, k, pos, f, axes=axes, layout=layout)
    assert torch.equal(qkv, before)
    check(a, q, pos, f, axes, layout), check(b, k, pos, f, axes, layout)
    c, e = kb.kroquant_rotary(q, k, pos, f, axes=axes, layout=layout, out=(q, k))
    assert c is q and e is k and torch.equal(q, a) and torch.equal(k, b)
    assert torch.equal(qkv[:, (H + KV) * d :], before[:, (H + KV) * d :])
    x = torch.randn(H, T, d, device="cuda", generator=g).to(dtype)       # heads first, broadcast over a batch of positions
    y = torch.zeros(T, H + 1, d + 8, device="cuda", dtype=dtype)
    kb.kroquant_rotary(x.transpose(0, 1), None, pos, f, axes=axes, layout=layout, out=y[:, 1:, 4 : 4 + d])
    check(y[:, 1:, 4 : 4 + d], x.transpose(0, 1), pos, f, axes, layout)
    assert bool((y[:, 0] == 0).all()) and bool((y[..., :4] == 0).all()) and bool((y[..., 4 + d :] == 0).all())
    one = x[:1].transpose(0, 1).expand(T, 5, d)                          # one head read five times
    check(kb.kroquant_rotary(one, None, pos, f, axes=axes, layout=layout), one, pos, f, axes, layout)


@pytest.mark.parametrize("shared", [True, False])
def test_batches(shared):
    B, T, H, d, axes = 3, 21, 4, 72, (24, 24, 24)
    g = gen(4)
    q, k = torch.randn(B, T, H, d, device="cuda", generator=g).bfloat16(), torch.randn(B, 2, T, d, device="cuda", generator=g).bfloat16().transpose(1, 2)
    pos = torch.randint(0, 99, (T, 3) if shared else (B, T, 3), device="cuda", generator=g, dtype=torch.int32)
    f = kb.rotary_frequencies(axes)
    a, b = kb.kroquant_rotary(q, k, pos, f, axes=axes)
    for i in range(B):
        p = pos if shared else pos[i]
        check(a[i], q[i], p, f, axes, "interleaved"), check(b[i], k[i], p, f, axes, "interleaved")


@pytest.mark.parametrize("B,T,H,d", [(700, 3, 2, 64), (1500, 1, 1, 64), (300, 7, 1, 71)])
def test_batches_of_few_tokens(B, T, H, d):
    """A CTA's tokens run over several batches."""
    g, axes = gen(B), (22, 20)
    x = torch.randn(T, B, H, d, device="cuda", generator=g).half().transpose(0, 1)
    for pos in (torch.randint(0, 999, (T, 2), device="cuda", generator=g, dtype=torch.int32), torch.randint(0, 999, (B, T, 2), device="cuda", generator=g, dtype=torch.int32)):
        f = kb.rotary_frequencies(axes)
        y, z = kb.kroquant_rotary(x, x.flip(2), pos, f, axes=axes, layout="half")
        every = pos.expand(B, T, 2).reshape(-1, 2)
        check(y.reshape(-1, H, d), x.reshape(-1, H, d), every, f, axes, "half")
        check(z.reshape(-1, H, d), x.flip(2).reshape(-1, H, d), every, f, axes, "half")


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_gradient_against_differences(layout):
    """sum(g * y(x)) is linear in x: its difference along h is sum(x_grad * h) up to 32-bit rounding of both sides."""
    T, H, d, axes = 13, 2, 40, (12, 20)
    g = gen(5)
    x, h, up = (torch.randn(T, H, d, device="cuda", generator=g) for _ in range(3))
    pos = torch.randint(0, 50, (T, 2), device="cuda", generator=g, dtype=torch.int32)
    f = kb.rotary_frequencies(axes)
    turn = lambda t, inverse=False: kb.kroquant_rotary(t, None, pos, f, axes=axes, layout=layout, inverse=inverse).double()  # noqa: E731
    difference = ((turn(x + h) - turn(x - h)) * up.double()).sum() / 2
    gradient = (turn(up, True) * h.double()).sum()
    # every term of the sums is off by at most 8 * 2^-24 of values below |x| + |h| <= 10
    assert abs(float(difference - gradient)) <= 8 * 2.0 ** -24 * 10 * float(up.abs().sum() + h.abs().sum())


def test_empty_other_stream_and_graph():
    f, pos = kb.rotary_frequencies((64,)), torch.arange(50, dtype=torch.int32, device="cuda")
    assert kb.kroquant_rotary(torch.empty(0, 4, 64, device="cuda"), None, pos[:0], f).shape == (0, 4, 64)
    x = torch.randn(50, 4, 64, device="cuda", generator=gen(6)).bfloat16()
    want = kb.kroquant_rotary(x, None, pos, f)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = kb.kroquant_rotary(x, None, pos, f, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = kb.kroquant_rotary(x, None, pos, f)
    x.neg_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, -want)


def test_not_finite_stays_in_its_pair():
    x = torch.randn(4, 2, 64, device="cuda", generator=gen(7))
    pos, f = torch.arange(4, dtype=torch.int32, device="cuda"), kb.rotary_frequencies((32,))
    want = kb.kroquant_rotary(x, None, pos, f)
    x[1, 0, 6], x[2, 1, 40] = float("nan"), float("inf")
    got = kb.kroquant_rotary(x, None, pos, f)
    assert bool(torch.isnan(got[1, 0, 6:8]).all()) and float(got[2, 1, 40]) == float("inf")
    same = torch.ones_like(x, dtype=torch.bool)
    same[1, 0, 6:8] = same[2, 1, 40] = False
    assert torch.equal(got[same], want[same])


def test_refusals():
    q, f, pos = torch.zeros(4, 2, 64, device="cuda"), kb.rotary_frequencies((64,)), torch.zeros(4, dtype=torch.int32, device="cuda")
    ok = dict(q=q, k=None, positions=pos, frequencies=f)
    kb.kroquant_rotary(**ok)
    for bad in (dict(q=q[0]), dict(q=q.double()), dict(q=q.transpose(1, 2)), dict(q=q.cpu()), dict(k=q.half()), dict(k=q[:3]), dict(k=q[..., :32]),
                dict(frequencies=f.float()), dict(frequencies=f.cpu()), dict(frequencies=f.repeat(2)), dict(positions=pos.long()), dict(positions=pos[:3]),
                dict(positions=pos.cpu()), dict(axes=(32, 30)), dict(axes=(33, 31)), dict(axes=(16, 16, 16, 8, 8)), dict(layout="other"),
                dict(axes=(32, 32)), dict(out=(q, q)), dict(k=q, out=q[:1]), dict(out=q[:, :1].expand(4, 2, 64)), dict(out=q.half()), dict(out=q[:3])):
        with pytest.raises(ValueError):
            kb.kroquant_rotary(**{**ok, **bad})
    big = torch.zeros(5, 2, 64, device="cuda")
    with pytest.raises(ValueError):                                      # shifted over its input
        kb.kroquant_rotary(big[:4], None, pos, f, out=big[1:])
    kb.kroquant_rotary(big[:2], None, pos[:2], f, out=big[2:4])


def test_outputs_keep_to_themselves():
    """out of q on k (or the other way round, or one out for both) would be read after it is written: refused.  Slices of one
    buffer lie between one another and share nothing."""
    g = torch.Generator(device="cuda")
    g.manual_seed(31)
    packed = torch.randn(37, 12, 64, device="cuda", generator=g).bfloat16()
    q, k = packed[:, :8], packed[:, 8:]
    pos, f = torch.arange(37, device="cuda", dtype=torch.int32), kb.rotary_frequencies((64,))
    want = kb.kroquant_rotary(q, k, pos, f)
    same = torch.zeros_like(q)
    for out in ((k.new_zeros(37, 8, 64), q[:, :4]), (same, same[:, :4])):
        with pytest.raises(ValueError):
            kb.kroquant_rotary(q, k, pos, f, out=out)
    with pytest.raises(ValueError):
        kb.kroquant_rotary(q[:, :4], k, pos, f, out=(k, torch.zeros_like(k)))
    got = kb.kroquant_rotary(q, k, pos, f, out=(q, k))
    assert torch.equal(got[0], want[0]) and torch.equal(packed[:, 8:], want[1])
