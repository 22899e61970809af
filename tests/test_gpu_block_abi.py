"""The block's operators through the C structs, against the same calls through the binding."""
import ctypes as C

import pytest
import torch

from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class NormProblem:
    """Inputs of the norm step and its backward pass; ``call`` fills the struct from its defaults and ``kw``."""

    def __init__(self, rows, d, seed):
        g = _gen(seed)
        self.rows, self.d = rows, d
        self.x, self.y, self.dn, self.dh = (torch.randn(rows, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(4))
        self.vectors = {k: torch.randn(d, device="cuda", generator=g) for k in ("gate", "weight", "scale", "shift")}

    def args(self, **kw):
        a = kb._NormArgs()
        kb.load_library().kroquant_norm_args_default(C.addressof(a))
        a.rows, a.d, a.norm, a.stream_dtype, a.branch_dtype, a.residual_scale = self.rows, self.d, 2, 1, 1, 0.5
        for k, v in self.vectors.items():
            setattr(a, k, v.data_ptr())
        for k in ("x", "y", "h", "n", "dn", "dh", "dx", "dy"):
            setattr(a, "ld_" + k, self.d)
        a.y = self.y.data_ptr()
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    def forward(self, **kw):
        h, n = torch.empty_like(self.x), torch.empty_like(self.x)
        a = self.args(x=self.x.data_ptr(), h=h.data_ptr(), n=n.data_ptr(), **kw)
        assert kb.load_library().kroquant_norm_residual(C.addressof(a), torch.cuda.current_stream().cuda_stream) == 0
        return h, n

    def backward(self, h, **kw):
        out = {k: torch.empty_like(self.x) for k in ("dx", "dy")}
        out.update({"d" + k: torch.empty(self.d, device="cuda") for k in self.vectors})
        a = self.args(h=h.data_ptr(), dn=self.dn.data_ptr(), dh=self.dh.data_ptr(), **{k: v.data_ptr() for k, v in out.items()}, **kw)
        L = kb.load_library()
        nbytes = L.kroquant_norm_residual_grad_scratch_bytes(C.addressof(a))
        scratch = torch.full((nbytes + 4096,), 77, device="cuda", dtype=torch.uint8)      # with canaries behind it
        assert L.kroquant_norm_residual_grad(C.addressof(a), scratch.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert bool((scratch[nbytes:] == 77).all())
        return out, nbytes


@pytest.mark.parametrize("rows,d", [(1, 640), (7, 640), (700, 640), (700, 256), (700, 2240), (37, 5600)])
@pytest.mark.parametrize("per", [2 ** 63 - 1, 2 ** 62, 2 ** 31])
def test_one_batch_of_any_number_of_rows(rows, d, per):
    p = NormProblem(rows, d, rows + d)
    want_h, want_n = kb.kroquant_norm_residual(p.x, p.y, norm="layer", residual_scale=0.5, **p.vectors)
    want = kb.kroquant_norm_residual_grad(p.dn, want_h, dh=p.dh, y=p.y, norm="layer", residual_scale=0.5, **p.vectors)
    h, n = p.forward(rows_per_batch=per)
    assert torch.equal(h, want_h) and torch.equal(n, want_n)
    got, _ = p.backward(h, rows_per_batch=per)
    assert set(got) == set(want)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("rows,d", [(700, 640), (700, 256), (700, 2240), (37, 5600)])
@pytest.mark.parametrize("per", [None, 3])
def test_shared_vectors_with_any_rows_per_batch(rows, d, per):
    """The default is 1 row per batch; without a stride the vectors are one for all rows, and so are the work and its bits."""
    p = NormProblem(rows, d, rows + d)
    want_h, want_n = kb.kroquant_norm_residual(p.x, p.y, norm="layer", residual_scale=0.5, **p.vectors)
    want = kb.kroquant_norm_residual_grad(p.dn, want_h, dh=p.dh, y=p.y, norm="layer", residual_scale=0.5, **p.vectors)
    kw = {} if per is None else {"rows_per_batch": per}
    h, n = p.forward(**kw)
    assert torch.equal(h, want_h) and torch.equal(n, want_n)
    got, nbytes = p.backward(h, **kw)
    assert nbytes == p.backward(h, rows_per_batch=rows)[1]
    for k in want:
        assert torch.equal(got[k], want[k]), k
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("M", [5, 100, 700])
@pytest.mark.parametrize("per", [None, 1, 3, 2 ** 63 - 1])
def test_linear_with_one_gate_row_and_any_rows_per_gate(M, per):
    """gate_stride 0: one row for all, whatever rows_per_gate says (its default is 1)."""
    N, K = 200, 288
    g = _gen(M)
    qa, sa = kb.kroquant_mxfp4_quantize(torch.randn(M, K, device="cuda", generator=g).to(torch.bfloat16), scale_layout="tiled")
    qw, sw = kb.kroquant_mxfp4_quantize(torch.randn(N, K, device="cuda", generator=g).to(torch.bfloat16), scale_layout="tiled")
    gate = torch.randn(N, device="cuda", generator=g)
    want = kb.kroquant_linear_mxfp4(qa, sa, qw, sw, gate=gate)
    e = kb._Epilogue()
    kb.load_library().kroquant_epilogue_default(C.addressof(e))
    e.gate, e.gate_dtype = gate.data_ptr(), 0
    if per is not None:
        e.rows_per_gate = per
    out = torch.empty_like(want)
    assert kb.load_library().kroquant_linear_mxfp4(qa.data_ptr(), sa.data_ptr(), qw.data_ptr(), sw.data_ptr(), M, N, K, C.addressof(e),
                                                   out.data_ptr(), 1, N, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, want)
    assert kb.kroquant_last_device_error() == 0
