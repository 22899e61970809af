"""CPU-only: what the block's entry points refuse before any CUDA call, and the layout helper of gated weights."""
import ctypes as C

import pytest
import torch

from paper_2607_21446_b200 import binding as kb

P = 4096                                     # a non-null, aligned address; nothing is launched


def linear(**kw):
    a = dict(a=P, sa=P, b=P, sb=P, M=8, N=64, K=64, e=None, out=P, dtype=1, ld=64)
    a.update(kw)
    e = a["e"]
    return kb.load_library().kroquant_linear_mxfp4(a["a"], a["sa"], a["b"], a["sb"], a["M"], a["N"], a["K"],
                                                   None if e is None else C.addressof(e), a["out"], a["dtype"], a["ld"], None)


def epilogue(**kw):
    e = kb._Epilogue()
    kb.load_library().kroquant_epilogue_default(C.addressof(e))
    for k, v in kw.items():
        setattr(e, k, v)
    return e


def norm(call="kroquant_norm_residual", **kw):
    a = kb._NormArgs()
    kb.load_library().kroquant_norm_args_default(C.addressof(a))
    for k, v in {**dict(rows=4, d=64, norm=1, x=P, ld_x=64, n=P, ld_n=64, h=P, ld_h=64, dn=P, ld_dn=64, dx=P, ld_dx=64), **kw}.items():
        setattr(a, k, v)
    fn = getattr(kb.load_library(), call)
    return fn(C.addressof(a), None) if call == "kroquant_norm_residual" else fn(C.addressof(a), None, 0, None)


def test_linear_refusals():
    assert linear(a=None) == 1 and linear(sb=None) == 1 and linear(out=None) == 1
    assert linear(M=-1) == 2 and linear(N=0) == 2 and linear(K=48) == 2 and linear(ld=63) == 2 and linear(M=1 << 25) == 2
    assert linear(e=epilogue(gate=P, gate_stride=32)) == 2 and linear(e=epilogue(gate=P, rows_per_gate=0)) == 2
    assert linear(e=epilogue(residual=P, residual_dtype=1, ld_residual=10)) == 2
    assert linear(a=P + 8) == 3 and linear(out=P + 1) == 3 and linear(e=epilogue(bias=P + 2)) == 3 and linear(e=epilogue(row_scale=P + 2)) == 3
    assert linear(dtype=3) == 5 and linear(e=epilogue(activation=9)) == 5 and linear(e=epilogue(glu=2)) == 5
    assert linear(e=epilogue(bias=P, bias_dtype=7)) == 5
    assert linear(M=0, out=None) == 0                                     # nothing to do


def test_grouped_refusals():
    L = kb.load_library()

    def grouped(offsets=P, experts=4, **kw):
        return L.kroquant_linear_mxfp4_grouped(P, P, P, P, offsets, experts, kw.get("M", 8), 64, 64, None, P, 1, 64, None)

    assert grouped(offsets=None) == 1 and grouped(experts=0) == 2 and grouped(experts=1025) == 2 and grouped(offsets=P + 2) == 3
    assert grouped(M=0) == 0


def test_norm_refusals():
    assert norm(x=None) == 1 and norm(n=None) == 1 and norm(norm=0, h=None) == 1
    assert norm(rows=-1) == 2 and norm(d=0) == 2 and norm(d=16385) == 2 and norm(ld_x=63) == 2 and norm(rows_per_batch=0) == 2
    assert norm(scale=P, scale_stride=32) == 2
    assert norm(x=P + 2) == 3 and norm(weight=P + 1) == 3
    assert norm(norm=3) == 5 and norm(stream_dtype=4) == 5 and norm(stream_dtype=1, branch_dtype=2) == 5
    assert norm(post_weight=P) == 5 and norm(norm=0, weight=P) == 5
    assert norm(rows=0, x=None) == 0
    grad = "kroquant_norm_residual_grad"
    assert norm(grad, h=None) == 1 and norm(grad, dn=None) == 1 and norm(grad, dx=None) == 1 and norm(grad, y=P, ld_y=64) == 1
    assert norm(grad, dx=P + 2) == 3 and norm(grad, ld_dn=1) == 2
    assert kb.load_library().kroquant_norm_residual_grad_scratch_bytes(None) == 0


@pytest.mark.parametrize("F", [1, 31, 32, 33, 100])
def test_interleave_glu(F):
    g, v = torch.randn(F, 5), torch.randn(F, 5)
    w = kb.interleave_glu(g, v)
    assert w.shape == (64 * ((F + 31) // 32), 5)
    for f in range(F):
        at = f // 32 * 64 + f % 32
        assert torch.equal(w[at], g[f]) and torch.equal(w[at + 32], v[f])
    filled = torch.zeros(w.shape[0], dtype=torch.bool)
    for f in range(F):
        filled[f // 32 * 64 + f % 32] = filled[f // 32 * 64 + f % 32 + 32] = True
    assert bool((w[~filled] == 0).all())
    assert torch.equal(kb.interleave_glu(g[:, 0], v[:, 0]), w[:, 0])
    with pytest.raises(ValueError):
        kb.interleave_glu(g, v[:, :4])
