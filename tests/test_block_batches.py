"""CPU-only: what the norm's backward pass makes of rows_per_batch.  Its scratch space holds three rows of d floats for every
(worker, batch) pair that can meet, so the size tells how many batches the call sees."""
import ctypes as C

import pytest

from paper_2607_21446_b200 import binding as kb

P = 4096                                     # a non-null, aligned address; nothing is launched


def scratch(**kw):
    a = kb._NormArgs()
    kb.load_library().kroquant_norm_args_default(C.addressof(a))
    for k, v in {**dict(rows=100, d=640, norm=2, h=P, ld_h=640, dn=P, ld_dn=640, dx=P, ld_dx=640, scale=P, dscale=P, weight=P, dweight=P), **kw}.items():
        setattr(a, k, v)
    return kb.load_library().kroquant_norm_residual_grad_scratch_bytes(C.addressof(a))


@pytest.mark.parametrize("stride", [0, 640])
@pytest.mark.parametrize("rows", [1, 3, 4, 5, 100, 20000])
@pytest.mark.parametrize("per", [2 ** 63 - 1, 2 ** 63 - 2, 2 ** 62, 2 ** 31])
def test_more_rows_per_batch_than_rows_is_one_batch(rows, per, stride):
    assert scratch(rows=rows, rows_per_batch=per, scale_stride=stride) == scratch(rows=rows, rows_per_batch=rows, scale_stride=stride) > 0


def test_batches_are_counted():
    one = scratch(rows=100, rows_per_batch=100, scale_stride=640)
    for per, batches in ((99, 2), (50, 2), (33, 4), (7, 15), (1, 100)):
        assert scratch(rows=100, rows_per_batch=per, scale_stride=640) == one + (batches - 1) * 3 * 640 * 4


@pytest.mark.parametrize("rows", [1, 100, 16384])
def test_shared_vectors_are_one_batch_whatever_rows_per_batch_says(rows):
    """(The default of rows_per_batch is 1.)"""
    assert scratch(rows=rows) == scratch(rows=rows, rows_per_batch=rows)
    assert scratch(rows=rows, rows_per_batch=7) == scratch(rows=rows, rows_per_batch=rows)
