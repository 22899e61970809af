"""Pages in ordinary use: short sequences under a table with room for long ones, and pages copied within a cache."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests.test_gpu_cache_attention import FORMATS, check, gen, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("d,group", [(72, 5), (128, 4), (128, 16), (256, 8)])
def test_short_sequences_under_a_wide_table(form, dtype, d, group):
    lengths = [300, 1, 0, 129, 511, 16]
    cache, table, n = make(lengths, 2, d, 16, form, dtype, d + group, width=512)
    q = torch.randn(len(lengths), 2 * group, d, device="cuda", generator=gen(d)).to(dtype)
    out, lse = kb.kroquant_cache_attention(q, cache, table, n, lse=True, out_dtype=torch.float32)
    check(out, q, cache, table, n, d ** -0.5, lse=lse)
    tight, its_lse = kb.kroquant_cache_attention(q, cache, table[:, :32], n, lse=True, out_dtype=torch.float32)
    check(tight, q, cache, table, n, d ** -0.5, lse=its_lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,heads,size", [(64, 3, 16), (128, 8, 7)])
def test_pages_copied_within_a_cache(dtype, d, heads, size):
    """Read into other pages, and written from them: a sequence that goes on from another's last page."""
    cache = kb.KVCache.empty(5, size, heads, d, "16bit", dtype)
    for t in (cache.k, cache.v):
        t.copy_(torch.randn(t.shape, device="cuda", generator=gen(size)))
    k, v = cache.k.clone(), cache.v.clone()
    offsets = torch.tensor([0, size], dtype=torch.int32, device="cuda")
    page = lambda i: torch.tensor([[i]], dtype=torch.int32, device="cuda")  # noqa: E731
    kb.kroquant_cache_read(cache, page(1), size, offsets=offsets, out=(cache.k[3].transpose(0, 1), cache.v[3].transpose(0, 1)))
    kb.kroquant_cache_write(cache, cache.k[2].transpose(0, 1), cache.v[2].transpose(0, 1), page(4), offsets=offsets)
    k[3], v[3], k[4], v[4] = k[1], v[1], k[2], v[2]
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
