"""Query heads that share a cache head do not touch one another, whatever their sizes, in the attention over the paged cache; tolerances as in
test_gpu_cache_attention.  A query enters the products over 8- and 4-bit caches as fp16 times a power of two: exact down to 2^-21 of its own
largest value."""
import math

import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests import cache_reference as cr
from tests.test_gpu_cache_attention import FORMATS, check, gen, make

pytestmark = pytest.mark.gpu
CODES = [f for f in FORMATS if f[0] != "16bit"]


def beyond(q, cache, table, lengths, scale):
    out = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for i, length in enumerate(lengths.tolist()):
        if length:
            k = cr.gather(cache, table[i], 0, length)[0].abs()
            terms = q[i].double().abs().view(cache.heads, -1, q.shape[2]) @ k.mT
            out[i] = (abs(scale) / math.log(2) * terms.amax(-1) >= 2.0 ** 127).view(-1)
    return out


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("group,d", [(4, 128), (7, 64), (16, 128), (12, 64), (9, 256), (40, 64)])
def test_a_query_that_is_not_finite_stays_with_its_head(form, dtype, group, d):
    for lengths in ([300, 33], [5000, 40]):                              # taken whole, and in parts
        cache, table, n = make(lengths, 2, d, 16, form, dtype, group)
        q = torch.randn(2, 2 * group, d, device="cuda", generator=gen(group)).to(dtype)
        clean = kb.kroquant_cache_attention(q, cache, table, n, out_dtype=torch.float32)
        bad = q.clone()
        bad[0, 1, 5], bad[0, 2, 7], bad[1, group, 0] = float("inf"), float("nan"), -float("inf")
        got, lse = kb.kroquant_cache_attention(bad, cache, table, n, out_dtype=torch.float32, lse=True)
        hit = torch.zeros(2, 2 * group, dtype=torch.bool, device="cuda")
        hit[0, 1] = hit[0, 2] = hit[1, group] = True
        assert not bool(torch.isfinite(got[hit]).any()) and not bool(torch.isfinite(lse[hit]).any())
        assert bool(torch.isfinite(got[~hit]).all()) and bool(torch.isfinite(lse[~hit]).all())
        check(torch.where(hit[..., None], clean, got), q, cache, table, n, d ** -0.5)


@pytest.mark.parametrize("form,dtype,loud", [(*f, loud) for f in CODES for loud in (6, 9, 14, 60, 120) if loud <= 14 or f[1] is torch.bfloat16])
@pytest.mark.parametrize("group", [3, 8, 16])
def test_heads_of_every_size(form, dtype, group, loud):
    """One head 2^loud times the others (as far as the type goes), one so much smaller."""
    cache, table, n = make([700, 129, 0], 2, 128, 16, form, dtype, loud)
    q = torch.randn(3, 2 * group, 128, device="cuda", generator=gen(loud)).clamp(-3, 3)
    q[:, 1] *= 2.0 ** loud
    q[:, group + 2] *= 2.0 ** -min(loud, 14 if dtype is torch.float16 else 60)
    q = q.to(dtype)
    for scale in (128 ** -0.5, -0.1, 0.0):
        out, lse = kb.kroquant_cache_attention(q, cache, table, n, out_dtype=torch.float32, lse=True, scale=scale)
        # A head with a score whose terms sum to 2^127 or more in units of log 2 has no statistics in 32 bits, whose largest number is 2^128: it is left out
        # (2^120 times 3 times keys of up to 16 in 128 channels is up to 2^133).
        keep = ~beyond(q, cache, table, n, scale)
        assert keep.sum() >= keep.numel() - 2
        zero = torch.where(keep[..., None], q, torch.zeros_like(q))
        instead, its_lse = kb.kroquant_cache_attention(zero, cache, table, n, out_dtype=torch.float32, lse=True, scale=scale)
        check(torch.where(keep[..., None], out, instead), zero, cache, table, n, scale, lse=torch.where(keep, lse, its_lse))


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_row_without_any_position_is_zero_whatever_its_query(form, dtype, value):
    cache, table, _ = make([100, 100, 100], 2, 64, 16, form, dtype, 6)
    table[0] = -1
    q = torch.randn(3, 4, 64, device="cuda", generator=gen(6)).to(dtype)
    q[0], q[1] = value, value
    n = torch.tensor([100, 0, 100], dtype=torch.int32, device="cuda")
    wide = torch.cat([table, torch.full((3, 3000), -1, dtype=torch.int32, device="cuda")], 1)
    longer = torch.tensor([40000, 0, 100], dtype=torch.int32, device="cuda")
    for t, lengths in ((table, n), (wide, n), (wide, longer)):
        out, lse = kb.kroquant_cache_attention(q, cache, t, lengths, lse=True)
        assert bool((out[:2] == 0).all()) and bool((lse[:2] == -math.inf).all())
        check(out[2:], q[2:], cache, t[2:], lengths[2:], 0.125, lse=lse[2:])
