"""kroquant_norm_residual and its backward pass against float64.

Tolerances, derived from the arithmetic: a 32-bit sum over a row is kept in at most 16 + 15 additions per path (a thread's
own values, two shuffle trees), so a statistic is off by at most 40 roundings of 2^-24 of the mean of its terms; with the
handful of roundings per element, every value before its output rounding is off by at most 64 * 2^-24 of the terms that
make it up.  Column sums over rows add one rounding per row.  Outputs are rounded once to their type.
"""
import numpy as np
import pytest
import torch

from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}
FLOOR = {torch.float32: 1e-30, torch.bfloat16: 1e-30, torch.float16: 2.0 ** -24}
EPS = 1e-6


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, dt, *shape, gain=1.0, mean=0.0):
    return (gain * torch.randn(*shape, device="cuda", generator=g) + mean).to(dt)


def _normal(v, kind):
    """-> (normalised, 1 / deviation, mean of the magnitudes / deviation)"""
    c = v - v.mean(1, keepdim=True) if kind == "layer" else v
    inv = 1 / (c.square().mean(1, keepdim=True) + EPS).sqrt()
    return c * inv, inv, v.abs().mean(1, keepdim=True) * inv


def _expand(v, rows, per, default):
    if v is None:
        return torch.full((1, 1), default, dtype=torch.float64, device="cuda")
    v = v.double()
    return v[None] if v.dim() == 1 else v.repeat_interleave(per, 0)[:rows]


def _forward(x, y, s, per):
    """float64 h, n and their tolerances before the output rounding."""
    rows = x.shape[0]
    h, th = s["residual_scale"] * x.double(), 0.0
    th = 64 * U * h.abs()
    if y is not None:
        gate, pw = _expand(s["gate"], rows, per, 1.0), _expand(s["post_weight"], rows, per, 1.0)
        r, size = y.double(), y.double().abs()
        if s["post_norm"] != "none":
            r, _, level = _normal(r, s["post_norm"])
            size = r.abs() + level
        h = h + gate * r * pw
        th = th + 64 * U * (gate * pw).abs() * size
    if s["norm"] == "none":
        return h, th, None, None
    m = _expand(s["weight"], rows, per, 1.0) * (1 + _expand(s["scale"], rows, per, 0.0))
    shift = _expand(s["shift"], rows, per, 0.0)
    xhat, inv, level = _normal(h, s["norm"])
    carried = inv * (th + th.mean(1, keepdim=True)) + xhat.abs() * (xhat.abs() * inv * th).mean(1, keepdim=True)
    return h, th, xhat * m + shift, m.abs() * (64 * U * (xhat.abs() + level) + carried) + 64 * U * shift.abs()


def _check(out, ref, tol):
    dt = out.dtype
    o = out.double()
    assert bool(torch.isfinite(o).all())
    worst = ((o - ref).abs() - (tol * (1 + ROUND[dt]) + ROUND[dt] * ref.abs() + FLOOR[dt])).max()
    assert float(worst) <= 0, float(worst)


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.float32, torch.bfloat16), (torch.float32, torch.float16),
         (torch.float32, torch.float32)]
WIDTHS = [1, 7, 8, 32, 200, 256, 257, 500, 512, 768, 1024, 1032, 1153, 2240, 4096, 5600, 8200, 12288, 16383, 16384]


def _case(rows, d, stream, branch, seed, batches=1, modulated=True, gated=True, norm="layer", post="none", vec=torch.float32):
    g = _gen(seed)
    s = dict(norm=norm, post_norm=post, residual_scale=0.75, eps=EPS)
    s["gate"] = _rand(g, vec, batches, d, gain=0.5) if gated else None
    s["post_weight"] = _rand(g, vec, d, gain=0.2, mean=1) if post != "none" else None
    s["weight"] = _rand(g, vec, d, gain=0.2, mean=1) if norm != "none" else None
    s["scale"] = _rand(g, vec, batches, d, gain=0.3) if modulated and norm != "none" else None
    s["shift"] = _rand(g, vec, batches, d, gain=0.3) if modulated and norm != "none" else None
    x, y = _rand(g, stream, rows, d, gain=2, mean=0.5), _rand(g, branch, rows, d, mean=-0.3)
    return x, y, s


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("norm,post", [("rms", "none"), ("layer", "rms"), ("rms", "layer"), ("none", "rms")])
def test_forward_of_every_width(d, norm, post):
    for (stream, branch), rows in zip(TYPES, (1, 5, 9, 3, 17)):
        x, y, s = _case(rows, d, stream, branch, d + rows, norm=norm, post=post)
        h, n = kb.kroquant_norm_residual(x, y, **s)
        ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, rows)
        _check(h, ref_h, tol_h)
        assert (n is None) == (norm == "none")
        if n is not None:
            _check(n, ref_n, tol_n)


@pytest.mark.parametrize("vec", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [96, 1153, 2240])
def test_batches_and_vector_types(vec, d):
    rows = 30
    for batches, per in ((3, 10), (5, 7), (30, 1), (4, 29)):
        x, y, s = _case(rows, d, torch.bfloat16, torch.bfloat16, d, batches, vec=vec)
        h, n = kb.kroquant_norm_residual(x, y, rows_per_batch=per, **s)
        ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, per)
        _check(h, ref_h, tol_h)
        _check(n, ref_n, tol_n)


@pytest.mark.parametrize("d", [1032, 2240, 4096, 4104, 5600, 12288, 16384])
@pytest.mark.parametrize("norm,post", [("rms", "none"), ("layer", "rms"), ("rms", "layer"), ("layer", "none"), ("none", "rms")])
def test_many_rows(d, norm, post):
    """Enough rows for persistent CTAs: several rows each, odd counts, batches that end inside a CTA's rows."""
    for (stream, branch), rows, batches, per in zip(TYPES, (1001, 701, 997, 650, 600), (1, 7, 997, 2, 3), (None, 101, 1, 333, 250)):
        x, y, s = _case(rows, d, stream, branch, d + rows, batches, norm=norm, post=post)
        h, n = kb.kroquant_norm_residual(x, y, rows_per_batch=per, **s)
        ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, per or rows)
        _check(h, ref_h, tol_h)
        if n is not None:
            _check(n, ref_n, tol_n)
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("rows", [147, 295, 296, 297, 445, 593])
@pytest.mark.parametrize("d,norm,post", [(1032, "layer", "rms"), (2240, "rms", "none"), (5600, "rms", "rms"), (16384, "layer", "layer")])
def test_about_as_many_rows_as_persistent_workers(rows, d, norm, post):
    """One row per worker, some with two, the last one with fewer than the others."""
    for stream, branch in TYPES[:2]:
        x, y, s = _case(rows, d, stream, branch, d + rows, 3, norm=norm, post=post)
        per = (rows + 2) // 3
        h, n = kb.kroquant_norm_residual(x, y, rows_per_batch=per, **s)
        ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, per)
        _check(h, ref_h, tol_h)
        _check(n, ref_n, tol_n)
    assert kb.kroquant_last_device_error() == 0


def test_many_rows_in_place_without_branch_and_vectors():
    x, y, s = _case(900, 2240, torch.bfloat16, torch.bfloat16, 3, post="rms")
    ref = _forward(x, y, s, 900)
    h, n = kb.kroquant_norm_residual(x, y, h_out=x, n_out=y, **s)
    assert h is x and n is y
    _check(h, *ref[:2])
    _check(n, *ref[2:])
    x = _rand(_gen(4), torch.float32, 800, 2240, mean=1000.0)
    _, n = kb.kroquant_norm_residual(x, norm="layer")
    c = x.double() - x.double().mean(1, keepdim=True)
    want = c / (c.square().mean(1, keepdim=True) + EPS).sqrt()
    assert float((n.double() - want).abs().max()) <= 64 * U * 1000 * 1.1


def test_without_branch_the_stream_is_handed_on():
    x, _, s = _case(12, 640, torch.bfloat16, torch.bfloat16, 5, gated=False)
    s["residual_scale"] = 1.0
    h, n = kb.kroquant_norm_residual(x, **s)
    assert h is x
    _check(n, *_forward(x, None, s, 12)[2:])
    s["residual_scale"] = 0.5
    h, n = kb.kroquant_norm_residual(x, branch_dtype=torch.bfloat16, **s)
    _check(h, *_forward(x, None, s, 12)[:2])


@pytest.mark.parametrize("d,pitch,shift", [(640, 640, 0), (640, 648, 8), (640, 647, 1), (641, 700, 3)])
def test_pitch_alignment_and_in_place(d, pitch, shift):
    rows = 21
    x, y, s = _case(rows, d, torch.bfloat16, torch.bfloat16, 6)
    bufs = [torch.full((shift + rows * pitch,), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = [b[shift:].view(rows, pitch)[:, :d] for b in bufs]
    views[0].copy_(x)
    views[1].copy_(y)
    h, n = kb.kroquant_norm_residual(views[0], views[1], h_out=views[0], n_out=views[1], **s)
    ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, rows)
    _check(h, ref_h, tol_h)
    _check(n, ref_n, tol_n)
    for b in bufs:
        assert bool((b[:shift] == 9).all()) and bool((b[shift:].view(rows, pitch)[:, d:] == 9).all())


def test_large_mean_keeps_its_variance():
    """Values around 1000 with deviation 1: the variance is taken about the mean."""
    x = _rand(_gen(7), torch.float32, 9, 4096, gain=1.0, mean=1000.0)
    _, n = kb.kroquant_norm_residual(x, norm="layer")
    c = x.double() - x.double().mean(1, keepdim=True)
    ref = c / (c.square().mean(1, keepdim=True) + EPS).sqrt()
    assert float((n.double() - ref).abs().max()) <= 64 * U * 1000 * 1.1


def _gradients(dn, dh, h, y, s, per):
    """float64 gradients and magnitudes of their terms."""
    rows, d = h.shape
    gate, pw = _expand(s["gate"], rows, per, 1.0), _expand(s["post_weight"], rows, per, 1.0)
    w, sc = _expand(s["weight"], rows, per, 1.0), _expand(s["scale"], rows, per, 0.0)
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731

    def back(g, hat, inv, kind, size):
        out = inv * (g - (mean(g) if kind == "layer" else 0) - hat * mean(g * hat))
        return out, inv * (size + mean(size) + hat.abs() * mean(size * hat.abs()))

    H, tH = (dh.double(), dh.double().abs()) if dh is not None else (torch.zeros_like(h, dtype=torch.float64),) * 2
    out, tol = {}, {}
    by_batch = lambda v: torch.stack([c.sum(0) for c in v.split(per)])  # noqa: E731
    if s["norm"] != "none":
        xhat, inv, level = _normal(h.double(), s["norm"])
        xs = xhat.abs() + level
        m = w * (1 + sc)
        add, size = back(dn.double() * m, xhat, inv, s["norm"], (dn.double() * m).abs())
        H, tH = H + add, tH + size * (1 + level)
        P, tP = dn.double() * xhat, dn.double().abs() * xs
        for name, val, t in (("weight", (1 + sc) * P, (1 + sc).abs() * tP),):
            if s[name] is not None:
                out["d" + name], tol["d" + name] = val.sum(0), t.sum(0)
        if s["scale"] is not None:
            out["dscale"], tol["dscale"] = by_batch(w * P), by_batch(w.abs() * tP)
        if s["shift"] is not None:
            out["dshift"], tol["dshift"] = by_batch(dn.double()), by_batch(dn.double().abs())
    out["dx"], tol["dx"] = s["residual_scale"] * H, s["residual_scale"] * tH
    if y is not None:
        yhat, yinv, ylevel, ys = y.double(), 1.0, 0.0, y.double().abs()
        if s["post_norm"] != "none":
            yhat, yinv, ylevel = _normal(y.double(), s["post_norm"])
            ys = yhat.abs() + ylevel
        if s["gate"] is not None:
            out["dgate"], tol["dgate"] = by_batch(H * yhat * pw), by_batch(tH * ys * pw.abs())
        if s["post_weight"] is not None:
            out["dpost_weight"], tol["dpost_weight"] = (gate * H * yhat).sum(0), (gate.abs() * tH * ys).sum(0)
        a, ta = gate * pw * H, (gate * pw).abs() * tH
        if s["post_norm"] != "none":
            a, size = back(a, yhat, yinv, s["post_norm"], ta)
            ta = size * (1 + ylevel)
        out["dy"], tol["dy"] = a, ta
    return out, tol


def _check_gradients(got, ref, tol, rows, vectors):
    assert set(got) == set(ref)
    for k in ref:
        r, t = ref[k], 128 * U * tol[k]
        if k not in ("dx", "dy"):
            t = (128 + rows) * U * tol[k]
            r, t = r.reshape(got[k].shape), t.reshape(got[k].shape)
            assert got[k].dtype == torch.float32 and got[k].shape == vectors[k[1:]].shape
        _check(got[k], r, t)


@pytest.mark.parametrize("d", [1, 8, 100, 256, 512, 513, 1024, 1153, 2240, 4608, 8192, 8200, 16384])
@pytest.mark.parametrize("norm,post", [("rms", "none"), ("layer", "none"), ("rms", "rms"), ("layer", "layer"), ("none", "layer")])
def test_backward_of_every_width(d, norm, post):
    for (stream, branch), rows in zip(TYPES, (1, 6, 40, 311, 2)):
        x, y, s = _case(rows, d, stream, branch, d + rows, norm=norm, post=post, modulated=rows != 40)
        g = _gen(1)
        dn = _rand(g, branch, rows, d) if norm != "none" else None
        dh = _rand(g, stream, rows, d)
        got = kb.kroquant_norm_residual_grad(dn, x, dh=dh, y=y, **s)
        _check_gradients(got, *_gradients(dn, dh, x, y, s, rows), rows, s)


@pytest.mark.parametrize("rows,batches,per", [(30, 3, 10), (30, 5, 7), (30, 30, 1), (1000, 7, 143), (999, 2, 500), (64, 4, 60)])
@pytest.mark.parametrize("d", [96, 1153, 2240])
def test_backward_with_batches(rows, batches, per, d):
    x, y, s = _case(rows, d, torch.bfloat16, torch.bfloat16, d, batches, post="rms")
    g = _gen(2)
    dn, dh = _rand(g, torch.bfloat16, rows, d), _rand(g, torch.bfloat16, rows, d)
    got = kb.kroquant_norm_residual_grad(dn, x, dh=dh, y=y, rows_per_batch=per, **s)
    ref, tol = _gradients(dn, dh, x, y, s, per)
    for k in ("dscale", "dshift", "dgate"):          # batches without rows have no gradient
        assert bool((got[k][ref[k].shape[0]:] == 0).all())
        ref[k] = torch.nn.functional.pad(ref[k], (0, 0, 0, batches - ref[k].shape[0]))
        tol[k] = torch.nn.functional.pad(tol[k], (0, 0, 0, batches - tol[k].shape[0]))
    _check_gradients(got, ref, tol, rows, s)


def test_backward_without_stream_gradient_branch_or_vectors():
    rows, d = 50, 640
    x, y, s = _case(rows, d, torch.bfloat16, torch.bfloat16, 8, gated=False, modulated=False)
    dn = _rand(_gen(3), torch.bfloat16, rows, d)
    _check_gradients(kb.kroquant_norm_residual_grad(dn, x, y=y, **s), *_gradients(dn, None, x, y, s, rows), rows, s)
    s["weight"] = None
    got = kb.kroquant_norm_residual_grad(dn, x, **s)
    assert set(got) == {"dx"}
    _check_gradients(got, *_gradients(dn, None, x, None, s, rows), rows, s)


@pytest.mark.parametrize("norm,post", [("rms", "layer"), ("layer", "rms"), ("layer", "none")])
def test_gradient_against_differences(norm, post):
    """<gradient, direction> against central differences of the forward kernel itself, in 32 bits.  Step 2^-6 along unit-size
    directions: the cubic remainder is below 1e-3 of the slope, the rounding of the sums below 1e-4 / step of it."""
    rows, d, step = 24, 640, 2.0 ** -6
    x, y, s = _case(rows, d, torch.float32, torch.float32, 9, 2, norm=norm, post=post)
    g = _gen(4)
    dn, dh = _rand(g, torch.float32, rows, d), _rand(g, torch.float32, rows, d)
    h, _ = kb.kroquant_norm_residual(x, y, **s)
    got = kb.kroquant_norm_residual_grad(dn, h, dh=dh, y=y, **s)

    def loss(x, y, s):
        h, n = kb.kroquant_norm_residual(x, y, **s)
        return float((h.double() * dh.double()).sum() + (n.double() * dn.double()).sum())

    for name in got:
        base = x if name == "dx" else y if name == "dy" else s[name[1:]]
        v = _rand(g, torch.float32, *base.shape)
        sides = []
        for sign in (1, -1):
            moved = base + sign * step * v
            if name == "dx":
                sides.append(loss(moved, y, s))
            elif name == "dy":
                sides.append(loss(x, moved, s))
            else:
                sides.append(loss(x, y, {**s, name[1:]: moved}))
        slope = (sides[0] - sides[1]) / (2 * step)
        want = float((got[name].double() * v.double()).sum())
        size = float(got[name].double().norm() * 1.0)
        assert abs(slope - want) <= 5e-3 * max(size, abs(want)), (name, slope, want, size)


def test_backward_is_deterministic_and_runs_on_another_stream():
    rows, d = 3000, 1152
    x, y, s = _case(rows, d, torch.bfloat16, torch.bfloat16, 10, 3, post="rms")
    dn, dh = _rand(_gen(5), torch.bfloat16, rows, d), _rand(_gen(6), torch.bfloat16, rows, d)
    first = kb.kroquant_norm_residual_grad(dn, x, dh=dh, y=y, **s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = [kb.kroquant_norm_residual_grad(dn, x, dh=dh, y=y, **s) for _ in range(3)]
    side.synchronize()
    for r in again:
        assert all(torch.equal(first[k], r[k]) for k in first)


@pytest.mark.parametrize("handle", [False, True])
def test_outputs_and_scratch_of_a_call_with_a_stream_belong_to_it(handle):
    """Memory freed on the current stream while its work is pending must not become the output or scratch of another stream's
    call, and what that call frees must not be taken by the current stream before the call has run."""
    rows, d = 2048, 1152
    x, y, s = _case(rows, d, torch.bfloat16, torch.bfloat16, 12, 2, post="rms")
    dn = _rand(_gen(7), torch.bfloat16, rows, d)
    want_h, want_n = kb.kroquant_norm_residual(x, y, **s)
    want = kb.kroquant_norm_residual_grad(dn, x, y=y, **s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    results = []
    for _ in range(4):
        results.append((kb.kroquant_norm_residual(x, y, stream=stream, **s), kb.kroquant_norm_residual_grad(dn, x, y=y, stream=stream, **s)))
        for _ in range(8):                                   # the current stream allocates and writes at once
            torch.full((rows, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    for (h, n), g in results:
        assert torch.equal(h, want_h) and torch.equal(n, want_n)
        assert all(torch.equal(g[k], want[k]) for k in want)


def test_masked_rows_and_non_finite_values_stay_in_their_rows():
    rows, d = 6, 512
    x, y, s = _case(rows, d, torch.float32, torch.float32, 11, post="rms")
    clean_h, clean_n = kb.kroquant_norm_residual(x, y, **s)
    x[1], y[1] = 0, 0                                    # a row of zeros
    x[3, 5], y[4, 7] = float("inf"), float("nan")
    h, n = kb.kroquant_norm_residual(x, y, **s)
    keep = [0, 2, 5]
    assert torch.equal(h[keep], clean_h[keep]) and torch.equal(n[keep], clean_n[keep])
    assert bool((h[1] == 0).all()) and torch.equal(n[1], s["shift"][0])
    assert not bool(torch.isfinite(n[3]).all()) and bool(torch.isnan(n[4]).all())


def test_empty_and_refused_calls():
    x, y, s = _case(8, 64, torch.bfloat16, torch.bfloat16, 12)
    f, b = kb.kroquant_norm_residual, kb.kroquant_norm_residual_grad
    h, n = f(x[:0], y[:0], **s)
    assert h.shape == (0, 64) and n.shape == (0, 64)
    got = b(y[:0], x[:0], y=y[:0], **s)
    assert all(float(got["d" + k].abs().max()) == 0 for k in ("weight", "scale", "shift", "gate"))
    n0 = kb.kroquant_launch_count()
    bad = [dict(norm="batch"), dict(gate=torch.ones(3, 64, device="cuda")), dict(weight=torch.ones(63, device="cuda")),
           dict(weight=torch.ones(64, device="cuda", dtype=torch.bfloat16), scale=torch.ones(64, device="cuda")),
           dict(scale=torch.ones(64)), dict(scale=torch.ones(2, 64, device="cuda"), shift=torch.ones(4, 64, device="cuda")),
           dict(scale=torch.ones(2, 64, device="cuda"), rows_per_batch=3), dict(h_out=x.float()), dict(n_out=x[:4])]
    for kw in bad:
        with pytest.raises(ValueError):
            f(x, y, **kw)
    for kw in (dict(post_weight=torch.ones(64, device="cuda")), dict(norm="none", weight=torch.ones(64, device="cuda"))):
        with pytest.raises(kb.KroQuantError):
            f(x, y, **kw)
    with pytest.raises(kb.KroQuantError):
        f(x, y.float())                                  # a 16-bit stream with a float branch
    with pytest.raises(kb.KroQuantError):
        f(torch.ones(2, 16385, device="cuda"))
    with pytest.raises(ValueError):
        f(x.t(), y.t())
    with pytest.raises(ValueError):
        b(None, x, y=y)
    with pytest.raises(ValueError):
        b(y, x, gate=torch.ones(64, device="cuda"))
    assert kb.kroquant_launch_count() == n0
