"""The norm's backward pass with many batches: a vector row for every row, or for every few, over more rows than there are workers.
Definitions and tolerances are those of test_gpu_norm."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests.test_gpu_norm import _case, _check_gradients, _forward, _check, _gen, _gradients, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [256, 640, 2240, 5600, 9001])
@pytest.mark.parametrize("rows,per", [(700, 1), (701, 2), (1999, 7)])
@pytest.mark.parametrize("post", ["none", "layer"])
def test_a_vector_row_for_every_few_rows(d, rows, per, post):
    batches = (rows + per - 1) // per
    x, y, s = _case(rows, d, torch.float32, torch.bfloat16, d + rows, batches, post=post)
    g = _gen(3)
    dn, dh = _rand(g, torch.bfloat16, rows, d), _rand(g, torch.float32, rows, d)
    h, n = kb.kroquant_norm_residual(x, y, rows_per_batch=per, **s)
    ref_h, tol_h, ref_n, tol_n = _forward(x, y, s, per)
    _check(h, ref_h, tol_h)
    _check(n, ref_n, tol_n)
    got = kb.kroquant_norm_residual_grad(dn, x, dh=dh, y=y, rows_per_batch=per, **s)
    _check_gradients(got, *_gradients(dn, dh, x, y, s, per), rows, s)
    assert kb.kroquant_last_device_error() == 0
