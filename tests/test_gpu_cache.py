"""The paged cache: what write leaves in the buffers against the formats' definitions (codes and scale bytes have to be equal), and
what read gives (one rounding to the type asked for; bf16 and float32 hold every cached value of these inputs exactly)."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests import cache_reference as cr

pytestmark = pytest.mark.gpu
FORMATS = ["16bit", "mxfp8", "mxfp4"]


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def filled(cache, byte=0x5A):
    for name in ("k", "v", "k_scales", "v_scales"):
        t = getattr(cache, name)
        if t is not None:
            t.view(torch.uint8).fill_(byte)
    return cache


def rows_of(n, heads, d, dtype, g):
    """Normal rows with loud channels, a zero row, blocks of very different size, and ties of both formats."""
    x = torch.randn(n, heads, d, generator=g)
    x[..., :: 7] *= 9
    x[0, 0] = 0
    if n > 2:
        x[1] *= 2.0 ** -12
        x[2, :, : min(d, 32)] = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])[torch.arange(min(d, 32)) % 8]
    return x.to(dtype)


def stored(cache, page, slot):
    """Buffers of one cell, all heads, as CPU tensors."""
    out = []
    for name in ("k", "v"):
        s = getattr(cache, name + "_scales")
        out.append((getattr(cache, name)[page, :, slot].cpu(), None if s is None else s[page, :, slot].cpu()))
    return out


def check_cell(cache, page, slot, k, v):
    for (codes, scales), x in zip(stored(cache, page, slot), (k, v)):
        d, C = cache.head_dim, 32 * ((cache.head_dim + 31) // 32)
        if cache.format == "16bit":
            assert torch.equal(codes[:, :d], x) and bool((codes[:, d:] == 0).all())
            continue
        _, want, byte = cr.quantized(x, cache.format)
        if cache.format == "mxfp4":
            want = want[..., 0::2] | (want[..., 1::2] << 4)
        assert torch.equal(codes, want.to(torch.uint8))
        assert torch.equal(scales[:, : C // 32], byte.to(torch.uint8)) and bool((scales[:, C // 32 :] == 0).all())


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,heads,size", [(128, 8, 16), (64, 1, 1), (72, 3, 7), (1, 2, 5), (31, 2, 16), (100, 5, 3), (129, 2, 4), (200, 1, 9), (256, 2, 64), (112, 20, 49)])
def test_one_row_per_sequence(form, dtype, d, heads, size):
    n, pages, width = 6, 17, 3
    g = gen(d + heads)
    cache = filled(kb.KVCache.empty(pages, size, heads, d, form, dtype))
    table = torch.randperm(pages, generator=g)[: width * 5].view(5, width)
    table = torch.cat([table, torch.tensor([[-1, pages, 2 ** 31 - 1]])]).to(torch.int32)             # the last sequence has no pages
    starts = torch.tensor([0, size - 1, size, width * size - 1, width * size, 0], dtype=torch.int32)  # the fifth lies beyond its table
    k, v = rows_of(n, heads, d, dtype, g), rows_of(n, heads, d, dtype, g)
    kb.kroquant_cache_write(cache, k.cuda(), v.cuda(), table.cuda(), starts=starts.cuda())
    touched = torch.zeros(pages, size, dtype=torch.bool)
    for i in range(4):
        page, slot = int(table[i, int(starts[i]) // size]), int(starts[i]) % size
        touched[page, slot] = True
        check_cell(cache, page, slot, k[i], v[i])
    for name in ("k", "v", "k_scales", "v_scales"):
        t = getattr(cache, name)
        if t is not None:
            assert bool((t.view(torch.uint8).cpu().transpose(1, 2)[~touched] == 0x5A).all()), name
    got_k, got_v = kb.kroquant_cache_read(cache, table.cuda(), n, starts=starts.cuda(), dtype=torch.float32)
    for got, x in ((got_k, k), (got_v, v)):
        want = x.float() if form == "16bit" else cr.quantized(x, form)[0].float()
        assert torch.equal(got[:4].cpu(), want[:4]) and bool((got[4:] == 0).all())
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("sizes,starts,size", [([5, 0, 1, 40], [3, 0, 63, 0], 16), ([0, 0, 7], [0, 9, 2], 1), ([300], [100], 7), ([1] * 70, list(range(70)), 8),
                                               ([3] * 1100, [0] * 1100, 4), ([64, 64, 64], None, 64)])
def test_ragged_rows(form, sizes, starts, size):
    heads, d, n = 2, 64, len(sizes)
    g = gen(n)
    need = [((starts[i] if starts else 0) + s + size - 1) // size for i, s in enumerate(sizes)]
    pages, width = sum(need) + 3, max(need) + 1
    order, at = torch.randperm(pages, generator=g).tolist(), 0
    table = torch.full((n, width), -1, dtype=torch.int32)
    for i, m in enumerate(need):
        table[i, :m] = torch.tensor(order[at : at + m], dtype=torch.int32)
        at += m
    before, behind = 3, 5
    offsets = before + torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(sizes).cumsum(0)])
    rows = int(offsets[-1]) + behind
    qkv = torch.randn(rows, 3, heads, d, generator=g).to(torch.bfloat16)
    k, v = qkv[:, 1], qkv[:, 2]                                          # slices of packed rows
    cache = filled(kb.KVCache.empty(pages, size, heads, d, form, torch.bfloat16))
    dev = dict(offsets=offsets.to(torch.int32).cuda(), starts=None if starts is None else torch.tensor(starts, dtype=torch.int32).cuda())
    packed = qkv.cuda()
    kb.kroquant_cache_write(cache, packed[:, 1], packed[:, 2], table.cuda(), **dev)
    for i in range(0, n, max(1, n // 5)):
        for r in range(0, sizes[i], max(1, sizes[i] // 3)):
            t = (starts[i] if starts else 0) + r
            check_cell(cache, int(table[i, t // size]), t % size, k[int(offsets[i]) + r], v[int(offsets[i]) + r])
    out = torch.full((rows, 2, heads, d + 1), 7.0, dtype=torch.bfloat16, device="cuda")               # element stores
    kb.kroquant_cache_read(cache, table.cuda(), rows, out=(out[:, 0, :, :d], out[:, 1, :, 1:]), **dev)
    for got, x in ((out[:, 0, :, :d], k), (out[:, 1, :, 1:], v)):
        want = x if form == "16bit" else cr.quantized(x, form)[0].to(torch.bfloat16)
        assert torch.equal(got[before : rows - behind].cpu(), want[before : rows - behind])
        assert bool((got[:before] == 7).all()) and bool((got[rows - behind :] == 7).all())
    again = kb.kroquant_cache_read(cache, table.cuda(), rows, **dev)
    assert again[0].dtype is torch.bfloat16 and torch.equal(again[0][before : rows - behind], out[before : rows - behind, 0, :, :d])
    assert bool((out[..., 0, :, d] == 7).all()) and bool((out[:, 1, :, 0] == 7).all())


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
def test_half_precision_out_and_extreme_blocks(form):
    """Blocks from the smallest to the largest bf16 magnitudes; float16 out rounds once and overflows to infinity."""
    e = torch.arange(-126, 128, 3)
    x = (1 + torch.rand(len(e), 1, 64, generator=gen(9))) * torch.exp2(e.double())[:, None, None].float() / 2
    x = x.to(torch.bfloat16)
    n = len(e)
    cache = kb.KVCache.empty(n, 1, 1, 64, form)
    table = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    kb.kroquant_cache_write(cache, x.cuda(), -x.cuda(), table)
    want = cr.quantized(x, form)[0]
    for dtype in (torch.float32, torch.float16):
        k, v = kb.kroquant_cache_read(cache, table, n, dtype=dtype)
        # 2^-127, the smallest scale, times half a unit lies below float32's normal range: flushed or not, within its smallest step
        assert bool(((k.cpu().double() - want.to(dtype).double()).abs().nan_to_num(0) <= 2.0 ** -126).all()) and torch.equal(k, -v)
        assert torch.equal(torch.isinf(k.cpu()), torch.isinf(want.to(dtype)))


def test_offsets_in_any_state_stay_inside():
    """Offsets that decrease, exceed the rows or are negative, and starts of any value: no row lands in a page that is not the table's."""
    heads, d, size, pages = 1, 32, 4, 12
    cache = filled(kb.KVCache.empty(pages, size, heads, d, "mxfp8"))
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32, device="cuda")
    x = torch.ones(20, heads, d, dtype=torch.bfloat16, device="cuda")
    for off in ([9, 4, 2, 30], [-5, 100, 3, 3], [2 ** 31 - 1, -2 ** 31, 0, 7], [0, 0, 0, 0]):
        for st in ([0, 0, 0], [-2 ** 31, 2 ** 31 - 1, 5]):
            args = dict(offsets=torch.tensor(off, dtype=torch.int32, device="cuda"), starts=torch.tensor(st, dtype=torch.int32, device="cuda"))
            kb.kroquant_cache_write(cache, x, x, table, **args)
            kb.kroquant_cache_read(cache, table, 20, **args)
    assert bool((cache.k[6:] == 0x5A).all()) and bool((cache.v_scales[6:] == 0x5A).all())


def test_cache_beyond_32_bit_offsets():
    heads, d, size = 8, 256, 64
    row = heads * size * d * 2
    pages = (5 << 30) // row
    k, v = (torch.empty(pages, heads, size, d, dtype=torch.float16, device="cuda") for _ in range(2))
    cache = kb.KVCache(k, v, head_dim=d, format="16bit")
    assert k.numel() * 2 > 1 << 32
    x = torch.randn(2 * size, heads, d, generator=gen(10)).half().cuda()
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 2 * size], dtype=torch.int32, device="cuda")
    kb.kroquant_cache_write(cache, x, x + 1, table, offsets=offsets)
    assert torch.equal(k[pages - 1], x[:size].transpose(0, 1)) and torch.equal(v[0], (x[size:] + 1).transpose(0, 1))
    a, b = kb.kroquant_cache_read(cache, table, 2 * size, offsets=offsets)
    assert torch.equal(a, x) and torch.equal(b, x + 1)


def test_streams_graph_and_empty_calls():
    cache = kb.KVCache.empty(8, 16, 2, 64, "mxfp4")
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    x = torch.randn(2, 2, 64, generator=gen(11)).to(torch.bfloat16).cuda()
    starts = torch.tensor([5, 40], dtype=torch.int32, device="cuda")
    kb.kroquant_cache_write(cache, x[:0], x[:0], table[:0])
    assert kb.kroquant_cache_read(cache, table[:0], 0)[0].shape == (0, 2, 64)
    kb.kroquant_cache_write(cache, x, x, table[:, :0])                    # a table without pages: nowhere to write
    assert bool((cache.k == 0).all())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    kb.kroquant_cache_write(cache, x, x, table, starts=starts, stream=s)
    a, _ = kb.kroquant_cache_read(cache, table, 2, starts=starts, stream=s)
    s.synchronize()
    want = cr.quantized(x.cpu(), "mxfp4")[0].to(torch.bfloat16)
    assert torch.equal(a.cpu(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kb.kroquant_cache_write(cache, x, x, table, starts=starts)
        b, _ = kb.kroquant_cache_read(cache, table, 2, starts=starts)
    starts.add_(1)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b.cpu(), 2 * want)
    assert torch.equal(kb.kroquant_cache_read(cache, table, 2, starts=starts - 1)[0].cpu(), want)


def test_refusals():
    c = kb.KVCache.empty(4, 8, 2, 64, "mxfp4")
    b = kb.KVCache.empty(4, 8, 2, 64, "16bit", torch.float16)
    table = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    kb.kroquant_cache_write(c, x, x, table)
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, kw in (((c, x[:2], x[:2], table), {}), ((c, x, x[:2], table), {}), ((c, x.float(), x.float(), table), {}), ((c, x, x.half(), table), {}),
                     ((b, x, x, table), {}), ((c, x[:, :1], x[:, :1], table), {}), ((c, x.cpu(), x.cpu(), table), {}), ((c, x, x, table.long()), {}),
                     ((c, x, x, table.cpu()), {}), ((c, x, x, table[0]), {}), ((c, x, x, table), dict(offsets=off[:3])), ((c, x, x, table), dict(offsets=off.long())),
                     ((c, x, x, table), dict(starts=off)), ((c, x, x, table), dict(starts=off[:3].cpu())), ((c, x.transpose(1, 2), x, table), {})):
        with pytest.raises(ValueError):
            kb.kroquant_cache_write(*args, **kw)
    for args, kw in (((c, table, 2), {}), ((c, table, 3), dict(dtype=torch.int32)), ((c, table, 3), dict(out=(x, x[:2]))), ((c, table, 3), dict(out=(x, x.half()))),
                     ((c, table, 3), dict(out=(x, x[:1].expand(3, 2, 64)))), ((c, table, 3), dict(out=(x, x.clone()), dtype=torch.float16))):
        with pytest.raises(ValueError):
            kb.kroquant_cache_read(*args, **kw)
