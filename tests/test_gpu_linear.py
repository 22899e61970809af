"""kroquant_linear_mxfp4 and kroquant_linear_mxfp4_grouped against float64 on the decoded operands.

Tolerance per element, derived from the arithmetic: the fp32 accumulation of exact products is off by at most
1e-6 sum|a||b| (the bound of the plain W4A4 product); bias, activation (slope at most 1.13, evaluation error at most
2^-20 |v|), the gated product, gate, row scale and residual each add a rounding of 2^-23 of their terms; the output is
rounded once to its type.
"""
import math

import numpy as np
import pytest
import torch

from oracle import c_oracle as co
from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu

OUT_ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}
OUT_FLOOR = {torch.float32: 1e-30, torch.bfloat16: 1e-30, torch.float16: 2.0 ** -24}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _quantized(rows, K, seed):
    """-> (codes, tiled scales, decoded float64); block scales spread over 2^-3 .. 2^3."""
    g = _gen(seed)
    x = torch.randn(rows, K, device="cuda", generator=g) / math.sqrt(K) * 4
    e = torch.randint(-3, 4, (rows, K // 32), device="cuda", generator=g).float()
    x = (x * torch.exp2(e).repeat_interleave(32, 1)).to(torch.bfloat16).contiguous()
    q, s = kb.kroquant_mxfp4_quantize(x, scale_layout="tiled")
    qr, sr = kb.kroquant_mxfp4_quantize(x)
    dec = torch.from_numpy(co.dequantize(qr.cpu().numpy(), sr.cpu().numpy()).astype(np.float64)).cuda()
    return q, s, dec


def _act64(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return v * 0.5 * torch.special.erfc(-v / math.sqrt(2))
    if act == "gelu_tanh":
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v


def _reference(a, w, N, act="none", glu=False, bias=None, gate=None, row_scale=None, residual=None, residual_scale=1.0):
    """float64 value and tolerance before the output rounding; gate already expanded to [M, N] or [N]."""
    v, tol = a @ w.t(), 1e-6 * (a.abs() @ w.abs().t())
    if bias is not None:
        v = v + bias.double()
        tol = tol + 2.0 ** -23 * (v.abs() + bias.double().abs())
    if glu:
        cols = torch.arange(N, device=v.device)
        first = cols // 32 * 64 + cols % 32
        f, tf = _act64(v[:, first], act), 1.13 * tol[:, first] + 2.0 ** -20 * v[:, first].abs()
        u, tu = v[:, first + 32], tol[:, first + 32]
        v, tol = f * u, f.abs() * tu + u.abs() * tf + tf * tu + 2.0 ** -23 * (f * u).abs()
    else:
        tol = 1.13 * tol + 2.0 ** -20 * v.abs()
        v = _act64(v, act)
    for factor in (gate, None if row_scale is None else row_scale[:, None]):
        if factor is not None:
            f = factor.double()
            v, tol = v * f, tol * f.abs() + 2.0 ** -23 * (v * f).abs()
    if residual is not None:
        r = residual_scale * residual.double()
        v, tol = v + r, tol + 2.0 ** -23 * (r.abs() + v.abs())
    return v, tol


def _check(out, ref, tol):
    dt = out.dtype
    o = out.double()
    assert bool(torch.isfinite(o).all())
    worst = ((o - ref).abs() - (tol * (1 + OUT_ROUND[dt]) + OUT_ROUND[dt] * ref.abs() + OUT_FLOOR[dt])).max()
    assert float(worst) <= 0, float(worst)


def _check_device():
    torch.cuda.synchronize()
    assert kb.kroquant_last_device_error() == 0


SHAPES = [(1, 32, 32), (1, 1, 64), (3, 160, 288), (32, 257, 1152), (33, 128, 256), (64, 2240, 1152), (65, 100, 5600), (127, 384, 512),
          (128, 256, 544), (129, 96, 288), (257, 513, 1152), (300, 512, 2240), (1000, 1057, 2240), (2049, 640, 4608)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_plain_product_of_every_size(M, N, K):
    qa, sa, a = _quantized(M, K, M + K)
    qw, sw, w = _quantized(N, K, N + K)
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, out_dtype=dt)
        _check(out, *_reference(a, w, N))
    _check_device()


@pytest.mark.parametrize("M,N,K", [(4099, 2001, 256), (6000, 1504, 1152)])
@pytest.mark.parametrize("residual", [False, True])
def test_several_tiles_per_cta(M, N, K, residual):
    """More tiles than the GPU runs at once: stages, scale slots and both accumulators go round."""
    qa, sa, a = _quantized(M, K, 41)
    qw, sw, w = _quantized(N, K, 42)
    bias = torch.randn(N, device="cuda", generator=_gen(43))
    for dt in (torch.float32, torch.bfloat16):
        res = torch.randn(M, N, device="cuda", generator=_gen(44)).to(dt) if residual else None
        for _ in range(3):
            out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, bias=bias, activation="silu", residual=res, out_dtype=dt)
        _check(out, *_reference(a, w, N, "silu", False, bias, residual=res))
    _check_device()


@pytest.mark.parametrize("glu", [False, True])
def test_several_tiles_per_cta_in_groups(glu):
    sizes, N, K = [2000, 0, 1500, 3000], 1504, 544
    R = 2 * N if glu else N
    qa, sa, a = _quantized(sum(sizes), K, 45)
    w = [_quantized(R, K, 46 + e) for e in range(4)]
    out = kb.kroquant_linear_mxfp4_grouped(qa, sa, torch.stack([x[0] for x in w]), torch.stack([x[1] for x in w]), _groups(sizes),
                                           activation="silu", glu=glu)
    lo = 0
    for e, n in enumerate(sizes):
        if n:
            _check(out[lo:lo + n], *_reference(a[lo:lo + n], w[e][2], N, "silu", glu))
        lo += n
    _check_device()


@pytest.mark.parametrize("M", [1, 40, 100, 700])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("glu", [False, True])
def test_activations_and_bias(M, act, glu):
    N, K = 333, 1152
    R = 64 * ((N + 31) // 32) if glu else N
    qa, sa, a = _quantized(M, K, 1)
    qw, sw, w = _quantized(R, K, 2)
    for dt, bdt in ((torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)):
        bias = torch.randn(R, device="cuda", generator=_gen(3)).to(bdt)
        out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, features=N, bias=bias, activation=act, glu=glu, out_dtype=dt)
        _check(out, *_reference(a, w, N, act, glu, bias))
    _check_device()


@pytest.mark.parametrize("M", [2, 200])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
def test_what_is_not_finite_stays_so(M, act):
    """NaN and infinity in a column: NaN stays NaN, +inf stays +inf, relu takes -inf to 0; other columns are untouched."""
    N, K = 96, 128
    qa, sa, a = _quantized(M, K, 51)
    qw, sw, w = _quantized(N, K, 52)
    bias = torch.zeros(N, device="cuda")
    bias[3], bias[40], bias[70] = float("nan"), float("inf"), float("-inf")
    out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, bias=bias, activation=act, out_dtype=torch.float32)
    assert bool(torch.isnan(out[:, 3]).all()) and bool((out[:, 40] == float("inf")).all())
    if act == "relu":
        assert bool((out[:, 70] == 0).all())
    rest = [c for c in range(N) if c not in (3, 40, 70)]
    ref, tol = _reference(a, w, N, act)
    _check(out[:, rest], ref[:, rest], tol[:, rest])
    _check_device()


@pytest.mark.parametrize("M,N", [(5, 64), (48, 320), (96, 101), (512, 512), (774, 577)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
def test_gate_row_scale_and_residual(M, N, dt):
    K = 544
    g = _gen(4)
    qa, sa, a = _quantized(M, K, 5)
    qw, sw, w = _quantized(N, K, 6)
    residual = torch.randn(M, N, device="cuda", generator=g).to(dt)
    row_scale = torch.rand(M, device="cuda", generator=g)
    bias = torch.randn(N, device="cuda", generator=g)
    for batches, per in ((0, None), (1, None), (3, (M + 2) // 3), (M, 1)):
        gate = None if batches == 0 else torch.randn(batches, N, device="cuda", generator=g).to(dt)
        out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, bias=bias, activation="gelu", gate=gate, rows_per_gate=per, row_scale=row_scale,
                                       residual=residual, residual_scale=0.5, out_dtype=dt)
        full = None if gate is None else gate.repeat_interleave(per or M, 0)[:M]
        _check(out, *_reference(a, w, N, "gelu", False, bias, full, row_scale, residual, 0.5))
    _check_device()


@pytest.mark.parametrize("M", [9, 400])
@pytest.mark.parametrize("shift,pitch", [(0, 0), (1, 7), (8, 8), (16, 40)])
def test_pitches_alignments_and_in_place_residual(M, shift, pitch):
    """out and residual at odd offsets and pitches, canaries around every row; out = the residual itself."""
    N, K = 200, 288
    qa, sa, a = _quantized(M, K, 7)
    qw, sw, w = _quantized(N, K, 8)
    flat = torch.full((shift + M * (N + pitch),), 77.0, dtype=torch.bfloat16, device="cuda")
    view = flat[shift:].view(M, N + pitch)[:, :N]
    res = torch.randn(M, N, device="cuda", generator=_gen(9)).to(torch.bfloat16)
    view.copy_(res)
    kb.kroquant_linear_mxfp4(qa, sa, qw, sw, residual=view, out=view)
    _check(view, *_reference(a, w, N, residual=res))
    assert bool((flat[:shift] == 77).all()) and bool((flat[shift:].view(M, N + pitch)[:, N:] == 77).all())
    _check_device()


def _groups(sizes):
    return torch.tensor([0] + list(np.cumsum(sizes)), dtype=torch.int32, device="cuda")


GROUPS = [[1], [0, 0, 1], [5, 0, 3, 0, 8], [32, 32], [64, 1, 63, 0], [127, 1, 128, 129], [0, 300, 0], [100] * 7, [1] * 40, [700, 0, 3, 513],
          [256, 256, 255, 257], [2000, 1]]


@pytest.mark.parametrize("sizes", GROUPS, ids=lambda s: "-".join(map(str, s[:6])))
@pytest.mark.parametrize("glu", [False, True])
def test_groups_of_every_size(sizes, glu):
    T, E, N, K = sum(sizes), len(sizes), 161, 544
    R = 64 * ((N + 31) // 32) if glu else N
    qa, sa, a = _quantized(T, K, 11)
    w = [_quantized(R, K, 20 + e) for e in range(E)]
    qw, sw = torch.stack([x[0] for x in w]), torch.stack([x[1] for x in w])
    bias = torch.randn(E, R, device="cuda", generator=_gen(12))
    row_scale = torch.rand(T, device="cuda", generator=_gen(13))
    offsets = _groups(sizes)
    for dt in (torch.float32, torch.bfloat16):
        out = kb.kroquant_linear_mxfp4_grouped(qa, sa, qw, sw, offsets, features=N, bias=bias, activation="silu", glu=glu,
                                               row_scale=row_scale, out_dtype=dt)
        lo = 0
        for e, n in enumerate(sizes):
            if n:
                _check(out[lo:lo + n], *_reference(a[lo:lo + n], w[e][2], N, "silu", glu, bias[e], None, row_scale[lo:lo + n]))
            lo += n
    _check_device()


@pytest.mark.parametrize("T", [20, 900])
def test_rows_outside_the_groups_and_wild_offsets(T):
    """Rows before the first and behind the last offset keep what they held; offsets outside [0, M] are clamped."""
    E, N, K = 3, 96, 288
    qa, sa, a = _quantized(T, K, 14)
    w = [_quantized(N, K, 30 + e) for e in range(E)]
    qw, sw = torch.stack([x[0] for x in w]), torch.stack([x[1] for x in w])
    for offsets, bounds in (([4, 9, 9, T - 3], [(4, 9), (9, 9), (9, T - 3)]), ([-7, 6, 11, 10 ** 9], [(0, 6), (6, 11), (11, T)]),
                            ([8, 3, 12, 12], [(8, 8), (3, 12), (12, 12)])):
        out = torch.full((T, N), 77.0, device="cuda")
        kb.kroquant_linear_mxfp4_grouped(qa, sa, qw, sw, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out)
        written = torch.zeros(T, dtype=torch.bool, device="cuda")
        for e, (lo, hi) in enumerate(bounds):
            if hi > lo:
                _check(out[lo:hi], *_reference(a[lo:hi], w[e][2], N))
                written[lo:hi] = True
        assert bool((out[~written] == 77).all())
    _check_device()


def test_many_experts_few_rows_each():
    E, N, K, T = 200, 64, 256, 333
    g = np.random.default_rng(3)
    sizes = np.bincount(g.integers(0, E, T), minlength=E).tolist()
    qa, sa, a = _quantized(T, K, 15)
    q1, s1, w1 = _quantized(E * 128, K, 16)                    # 128 rows per expert: the tiled scales split evenly
    qw, sw = q1.view(E, 128, K // 2)[:, :N].contiguous(), s1.view(E, -1)
    out = kb.kroquant_linear_mxfp4_grouped(qa, sa, qw, sw, _groups(sizes), out_dtype=torch.float32)
    lo = 0
    for e, n in enumerate(sizes):
        if n:
            _check(out[lo:lo + n], *_reference(a[lo:lo + n], w1.view(E, 128, K)[e, :N], N))
        lo += n
    _check_device()


@pytest.mark.parametrize("M,E", [(24, 1), (200, 1), (1000, 1), (96, 6), (1500, 3)])
def test_same_bits_every_time_and_on_another_stream(M, E):
    N, K = 640, 2240
    qa, sa, _ = _quantized(M, K, 17)
    q1, s1, _ = _quantized(E * N, K, 18)
    qw, sw = q1.view(E, N, K // 2), s1.view(E, -1)
    offsets = _groups([M // E] * E)

    def call():
        if E == 1:
            return kb.kroquant_linear_mxfp4(qa, sa, qw[0], sw[0], activation="silu")
        return kb.kroquant_linear_mxfp4_grouped(qa, sa, qw, sw, offsets, activation="silu")

    first = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        outs = [call() for _ in range(5)]
    side.synchronize()
    assert all(torch.equal(first, o) for o in outs)
    _check_device()


def test_dense_equals_one_group_and_the_existing_product():
    M, N, K = 512, 384, 1152
    qa, sa, _ = _quantized(M, K, 19)
    qw, sw, _ = _quantized(N, K, 20)
    dense = kb.kroquant_linear_mxfp4(qa, sa, qw, sw)
    assert torch.equal(dense, kb.kroquant_linear_mxfp4_grouped(qa, sa, qw[None], sw[None], _groups([M])))
    assert torch.equal(dense, kb.kroquant_gemm_mxfp4(qa, sa, qw, sw))


def test_captured_in_a_graph():
    M, N, K = 48, 256, 1152
    qa, sa, a = _quantized(M, K, 21)
    qw, sw, w = _quantized(N, K, 22)
    out = torch.zeros(M, N, device="cuda")
    kb.kroquant_linear_mxfp4(qa, sa, qw, sw, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kb.kroquant_linear_mxfp4(qa, sa, qw, sw, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    _check(out, *_reference(a, w, N))


def test_interleave_glu_is_what_the_layer_reads():
    F, K, M = 70, 64, 10
    wg = torch.randn(F, K, device="cuda", generator=_gen(23)).to(torch.bfloat16)
    wu = torch.randn(F, K, device="cuda", generator=_gen(24)).to(torch.bfloat16)
    qw, sw = kb.kroquant_mxfp4_quantize(kb.interleave_glu(wg, wu), scale_layout="tiled")
    qa, sa, a = _quantized(M, K, 25)
    out = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, features=F, activation="silu", glu=True, out_dtype=torch.float32)
    parts = []
    for w in (wg, wu):
        q, s = kb.kroquant_mxfp4_quantize(w)
        parts.append(a @ torch.from_numpy(co.dequantize(q.cpu().numpy(), s.cpu().numpy()).astype(np.float64)).cuda().t())
    ref = _act64(parts[0], "silu") * parts[1]
    assert float((out.double() - ref).abs().max()) <= 1e-5 * float(ref.abs().max())


def test_empty_and_refused_calls():
    M, N, K = 64, 96, 288
    qa, sa, _ = _quantized(M, K, 26)
    qw, sw, _ = _quantized(N, K, 27)
    f = kb.kroquant_linear_mxfp4
    assert f(qa[:0], sa[:0], qw, sw).shape == (0, N)
    n0 = kb.kroquant_launch_count()
    ones = torch.ones(N, device="cuda")
    bad = [dict(activation="swish"), dict(bias=ones[:-1]), dict(gate=torch.ones(5, N, device="cuda")), dict(features=N - 1), dict(glu=True),
           dict(gate=torch.ones(2, N, device="cuda"), rows_per_gate=31), dict(row_scale=torch.ones(M, device="cuda", dtype=torch.float16)),
           dict(residual=torch.ones(M, N + 1, device="cuda")), dict(residual=torch.ones(N, M, device="cuda").t()),
           dict(out=torch.ones(M, N, device="cuda", dtype=torch.float64)), dict(out_dtype=torch.int32), dict(bias=ones.cpu())]
    for kw in bad:
        with pytest.raises((ValueError, KeyError)):
            f(qa, sa, qw, sw, **kw)
    with pytest.raises(ValueError):
        f(qa, sa[:-1], qw, sw)
    with pytest.raises(ValueError):
        f(qa, sa, qw[:, :-1].contiguous(), sw)
    g = kb.kroquant_linear_mxfp4_grouped
    for offsets in (None, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"),
                    torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            g(qa, sa, qw[None], sw[None], offsets)
    L = kb.load_library()
    out = torch.empty(M, N, device="cuda")
    args = [qa.data_ptr(), sa.data_ptr(), qw.data_ptr(), sw.data_ptr(), M, N, K, None, out.data_ptr(), 0, N, None]

    def status(**kw):
        a = list(args)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return L.kroquant_linear_mxfp4(*a)

    assert status(_0=None) == 1 and status(_8=None) == 1
    assert status(_6=K + 16) == 2 and status(_5=0) == 2 and status(_4=-1) == 2 and status(_10=N - 1) == 2
    assert status(_0=qa.data_ptr() + 8) == 3 and status(_8=out.data_ptr() + 2) == 3
    assert status(_9=7) == 5
    assert kb.kroquant_launch_count() == n0
