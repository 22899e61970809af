"""Products of 16-bit rows with MXFP4 weights against 64 bits.  Tolerance before the epilogue: the weight's values and x are exact, the
fp32 sums of K products lose at most (K / 16 + 16) 2^-23 of sum |x w| (16 products a step of the tensor core, truncated); x below 2^-28 of the largest of
its 128 channels is off by 2^-40 of that.  The activations have slopes up to 1.13 and are good to 2^-20 of their value; one rounding to out's type."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests import cache_reference as cr

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def weight(rows, K, g, spread=True):
    w = torch.randn(rows, K, device="cuda", generator=g) * K ** -0.5
    if spread:
        w *= torch.exp2(torch.randint(-6, 7, (rows, K // 32), device="cuda", generator=g).float()).repeat_interleave(32, 1)
    q, s = kb.kroquant_mxfp4_quantize(w.bfloat16(), scale_layout="tiled")
    _, plain = kb.kroquant_mxfp4_quantize(w.bfloat16())
    return q, s, cr.decoded(q, plain, "mxfp4", K)


def act(v, name):
    return {"none": lambda z: z, "relu": lambda z: z.clamp_min(0), "silu": lambda z: z * torch.sigmoid(z),
            "gelu": lambda z: 0.5 * z * torch.special.erfc(-z / 2 ** 0.5),
            "gelu_tanh": lambda z: z * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3))}[name](v)


def expected(x, w, N, bias=None, activation="none", glu=False, gate=None, rows_per_gate=None, row_scale=None, residual=None, residual_scale=1.0):
    """-> value and tolerance without out's rounding"""
    K = x.shape[1]
    v, size = x.double() @ w.T, x.double().abs() @ w.abs().T
    tol = (K / 16 + 16) * 2.0 ** -23 * size + 2.0 ** -40 * x.abs().amax(1, keepdim=True).double() * w.abs().sum(1)
    if bias is not None:
        v = v + bias.double()
        tol = tol + 2.0 ** -24 * (size + bias.double().abs())
    if glu:
        cols = torch.arange(N, device="cuda")
        at = cols // 32 * 64 + cols % 32
        a, b = act(v[:, at], activation), v[:, at + 32]
        slope = 1.13 if activation != "none" else 1.0
        tol = (slope * tol[:, at] + 2.0 ** -20 * a.abs()) * (b.abs() + tol[:, at + 32]) + a.abs() * tol[:, at + 32] + 2.0 ** -23 * (a * b).abs()
        v = a * b
    else:
        v = act(v, activation)
        tol = 1.13 * tol + 2.0 ** -20 * v.abs()
    for f in (None if gate is None else gate.double().view(-1, N).repeat_interleave(rows_per_gate or x.shape[0], 0)[: x.shape[0]],
              None if row_scale is None else row_scale.double()[:, None]):
        if f is not None:
            v, tol = v * f, tol * f.abs() + 2.0 ** -23 * (v * f).abs()
    if residual is not None:
        v, tol = residual_scale * residual.double() + v, tol + 2.0 ** -22 * (residual_scale * residual.double()).abs() + 2.0 ** -23 * v.abs()
    return v, tol


def check(out, want, tol):
    tol = tol + torch.finfo(out.dtype).eps / 2 * (want.abs() + tol) + torch.finfo(out.dtype).smallest_normal
    over = (out.double() - want).abs() - tol
    assert bool((over <= 0).all()), float(over.max())
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", [(1, 6912, 1152), (1, 1, 32), (2, 127, 96), (5, 129, 160), (8, 256, 128), (9, 33, 4096), (16, 4608, 12288), (17, 1000, 2240),
                                   (33, 31, 288), (64, 640, 5600), (3, 12288, 4608), (1, 40, 65536), (16, 100, 40000), (7, 20000, 64)])
def test_sizes(dtype, M, N, K):
    g = gen(M + N)
    q, s, w = weight(N, K, g)
    x = torch.randn(M, K, device="cuda", generator=g)
    x[:, torch.randint(0, K, (max(1, K // 50),), device="cuda", generator=g)] *= 50
    x = x.to(dtype)
    want, tol = expected(x, w, N)
    check(kb.kroquant_linear_w4a16(x, q, s, out_dtype=torch.float32), want, tol)
    check(kb.kroquant_linear_w4a16(x, q, s), want, tol)


@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 100, 288), (6, 704, 1152), (20, 65, 640)])
def test_epilogue(activation, glu, M, N, K):
    g = gen(N)
    R = 64 * ((N + 31) // 32) if glu else N
    q, s, w = weight(R, K, g, spread=False)
    x = torch.randn(M, K, device="cuda", generator=g).bfloat16()
    bias = torch.randn(R, device="cuda", generator=g).half()
    gate = torch.randn(2, N, device="cuda", generator=g).bfloat16()
    row_scale = torch.rand(M, device="cuda", generator=g)
    residual = torch.randn(M, N + 3, device="cuda", generator=g).half()[:, 1 : N + 1]
    full = dict(bias=bias, activation=activation, glu=glu, gate=gate, rows_per_gate=(M + 1) // 2, row_scale=row_scale, residual=residual, residual_scale=0.5)
    for kw in (dict(activation=activation, glu=glu), dict(activation=activation, glu=glu, bias=bias.float()), full):
        want, tol = expected(x, w, N, **kw)
        for dt in (torch.float32, torch.float16):
            check(kb.kroquant_linear_w4a16(x, q, s, features=N, out_dtype=dt, **kw), want, tol)
    out = residual.clone()
    check(kb.kroquant_linear_w4a16(x, q, s, features=N, **{**full, "residual": out, "out": out}), *expected(x, w, N, **full))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K,glu", [(1, 2150, 4096, False), (4, 2113, 4128, False), (8, 2049, 8192, True), (16, 1050, 4160, True), (20, 1150, 6144, False),
                                       (64, 600, 4608, False), (33, 2305, 12320, False)])
def test_long_rows_and_many_tiles(dtype, M, N, K, glu):
    """Odd and even numbers of tiles of 128 weight rows, where K is long and the tiles are many, but all run at once."""
    g = gen(M + N + 1)
    R = 64 * ((N + 31) // 32) if glu else N
    q, s, w = weight(R, K, g)
    x = torch.randn(M, K, device="cuda", generator=g).to(dtype)
    residual = torch.randn(M, N, device="cuda", generator=g).to(dtype)
    kw = dict(bias=torch.randn(R, device="cuda", generator=g), glu=glu, activation="silu" if glu else "none", residual=residual)
    want, tol = expected(x, w, N, **kw)
    check(kb.kroquant_linear_w4a16(x, q, s, features=N, out_dtype=torch.float32, **kw), want, tol)
    guard = torch.full((M + 2, N), 7.0, device="cuda", dtype=dtype)
    out = kb.kroquant_linear_w4a16(x, q, s, features=N, out=guard[1:-1], **kw)
    check(out, want, tol)
    assert bool((guard[0] == 7).all()) and bool((guard[-1] == 7).all())
    assert torch.equal(out, kb.kroquant_linear_w4a16(x, q, s, features=N, out_dtype=dtype, **kw))


@pytest.mark.parametrize("offset,pitch", [(0, 296), (1, 289), (8, 304), (4, 292)])
def test_rows_with_a_pitch(offset, pitch):
    g = gen(pitch)
    q, s, w = weight(200, 288, g)
    room = torch.full((5, pitch + 9), float("nan"), device="cuda", dtype=torch.float16)[:, :pitch]
    x = room[:, offset : offset + 288] if offset + 288 <= pitch else room[:, :288]
    x.copy_(torch.randn(5, 288, device="cuda", generator=g))
    out = torch.full((5, 203), 7.0, device="cuda")
    check(kb.kroquant_linear_w4a16(x, q, s, out=out[:, 2:202]), *expected(x, w, 200))
    assert bool((out[:, :2] == 7).all()) and bool((out[:, 202:] == 7).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_unequal_channels(dtype):
    """Rows of every size within the type, channels 2^20 apart, zero rows, and blocks of weights 2^30 apart."""
    g = gen(60)
    K, N = 640, 96
    q, s, _ = weight(N, K, g)
    s = s.view(-1, 32, 4, 4)
    s += torch.randint(0, 30, s.shape, device="cuda", generator=g, dtype=torch.uint8)
    plain = s.permute(0, 2, 1, 3).reshape(-1, 128, 4)                    # [K tile][row][block]; N <= 128: one row tile
    byte = plain.permute(1, 0, 2).reshape(128, -1)[:N, : K // 32]
    w = cr.decoded(q, byte, "mxfp4", K)
    top = 6 if dtype is torch.float16 else 60
    x = torch.randn(8, K, device="cuda", generator=g) * torch.exp2(torch.randint(-14, top, (8, 1), device="cuda", generator=g).float())
    x[:, 5::64] *= 2.0 ** (-8 if dtype is torch.float16 else -20)
    x[3] = 0
    x = x.to(dtype)
    check(kb.kroquant_linear_w4a16(x, q, s.reshape(-1), out_dtype=torch.float32), *expected(x, w, N))


def test_not_finite_rows_stay_rows():
    g = gen(61)
    q, s, _ = weight(64, 256, g)
    x = torch.randn(10, 256, device="cuda", generator=g).bfloat16()
    want = kb.kroquant_linear_w4a16(x, q, s)
    x[2, 7], x[9, 200] = float("nan"), float("inf")
    got = kb.kroquant_linear_w4a16(x, q, s)
    keep = [0, 1, 3, 4, 5, 6, 7, 8]
    assert torch.equal(got[keep], want[keep]) and not bool(torch.isfinite(got[[2, 9]]).any())


def test_rows_do_not_depend_on_their_neighbours_and_calls_repeat():
    g = gen(62)
    q, s, _ = weight(1000, 2240, g)
    x = torch.randn(64, 2240, device="cuda", generator=g).bfloat16()
    for M in (1, 8, 16, 64):
        a, b = kb.kroquant_linear_w4a16(x[:M], q, s), kb.kroquant_linear_w4a16(x[:M], q, s)
        assert torch.equal(a, b)
        flipped = x[:M].flip(0).contiguous()
        assert torch.equal(kb.kroquant_linear_w4a16(flipped, q, s).flip(0), a)


def test_stream_and_graph():
    g = gen(63)
    q, s, _ = weight(512, 1152, g)
    x = torch.randn(4, 1152, device="cuda", generator=g).bfloat16()
    want = kb.kroquant_linear_w4a16(x, q, s)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = kb.kroquant_linear_w4a16(x, q, s, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = kb.kroquant_linear_w4a16(x, q, s)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, 2 * want)


def test_layer_for_a_few_rows():
    """LinearW4A4.few: the transform in X's type, then the product with the layer's own weight."""
    from examples.quantized_block import dense_layer
    g = gen(64)
    layer = dense_layer((torch.randn(640, 1152, device="cuda", generator=g) * 0.03).bfloat16())
    X = torch.randn(5, 1152, device="cuda", generator=g).bfloat16()
    bias = torch.randn(640, device="cuda", generator=g)
    turned = kb.kroquant_quantize_dual(X, layer.factors)[2]
    want = kb.kroquant_linear_w4a16(turned, layer.w_codes, layer.w_scales, bias=bias, activation="gelu")
    assert torch.equal(layer.few(X, bias=bias, activation="gelu"), want)
    with pytest.raises(ValueError):
        layer.few(X[:, :1120].contiguous())
    with pytest.raises(ValueError):
        layer.few(X.repeat(13, 1))


def test_refusals():
    g = gen(65)
    q, s, _ = weight(64, 256, g)
    x = torch.zeros(3, 256, device="cuda", dtype=torch.bfloat16)
    assert kb.kroquant_linear_w4a16(x[:0], q, s).shape == (0, 64)
    for args, kw in (((x.float(), q, s), {}), ((x[0], q, s), {}), ((x[:, :224], q, s), {}), ((x.t(), q, s), {}), ((x.cpu(), q, s), {}), ((x, q.cpu(), s), {}),
                     ((x, q, s[:-16]), {}), ((x.repeat(22, 1), q, s), {}), ((x, q, s), dict(features=63)), ((x, q, s), dict(activation="tanh")),
                     ((x, q, s), dict(bias=torch.zeros(63, device="cuda"))), ((x, q, s), dict(out=torch.zeros(3, 63, device="cuda"))),
                     ((x, q, s), dict(row_scale=torch.zeros(4, device="cuda"))), ((x, q, s), dict(out_dtype=torch.int8))):
        with pytest.raises(ValueError):
            kb.kroquant_linear_w4a16(*args, **kw)
