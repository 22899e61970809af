"""Attention over the paged cache against softmax in 64 bits over the values the cache holds.

Tolerance of a value sum_t w_t v_t (w normalised): the weights enter the product rounded to 11 bits (half a step 2^-11 relative; bf16
caches: two bf16 terms, 2^-17), the exponential is good to 2^-22, and a score that is off by delta turns w by delta: fp32 sums of C
products lose at most (C / 16 + 8) 2^-23 of scale * sum |q k| (16 products a step of the tensor core, truncated, and the factors).  So
    |out - exact| <= (2^-11 + 2^-21 + 2 delta) sum_t w_t |v_t| + half a step of out's type,
and the sum over positions adds (T / 16 + 8) 2^-23 in the worst case.

Weights enter as fp16(w 2^9 2^(S - R)), w relative to a reference that is the largest weight or up to 2^6 below it, S and R scale bytes (1 for 16-bit
values), with fp16's smallest step 2^-24: one rounds by up to 2^-25, that is 2^-34 of the reference, times a code of at most 6 (448) units of R, where
the largest value has at least 4 (256): 1.75 max |v|; the sum they are divided by is at least 1, the reference's own weight.  Where the
positions that count hold zeros in a channel this is all there is: 2^-34 * 1.75 T max |v| more (not with bf16 values)."""
import math

import pytest
import torch

from paper_2607_21446_b200 import binding as kb
from tests import cache_reference as cr

pytestmark = pytest.mark.gpu
FORMATS = [("16bit", torch.bfloat16), ("16bit", torch.float16), ("mxfp8", torch.bfloat16), ("mxfp4", torch.bfloat16), ("mxfp4", torch.float16)]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make(lengths, heads, d, size, form, dtype, seed, spare=2, width=None, gain=1.0):
    """A cache whose pages hold garbage (NaN where the format has it) but at the sequences' positions; pages in random order."""
    g = gen(seed)
    need = [(n + size - 1) // size for n in lengths]
    width = max(need + [1]) if width is None else width
    pages = sum(need) + spare
    cache = kb.KVCache.empty(pages, size, heads, d, form, dtype)
    C = 32 * ((d + 31) // 32)
    for name in ("k", "v"):
        t = getattr(cache, name)
        t.view(torch.uint8).fill_(0xFF)                                  # NaN in bf16, fp16 and E4M3, -6 in E2M1
        s = getattr(cache, name + "_scales")
        if s is not None:
            s.fill_(0xFF)
    order, at = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist(), 0
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    for i, m in enumerate(need):
        table[i, :m] = torch.tensor(order[at : at + m], dtype=torch.int32)
        at += m
    rows = sum(lengths)
    if rows:
        x = torch.randn(2, rows, heads, d, device="cuda", generator=g)
        x[0, ..., :: 11] *= 5
        x[1] *= 0.5 * torch.exp2(torch.randint(-3, 4, (rows, heads, 1), device="cuda", generator=g).float())   # positions of unequal size
        x = (x * gain).to(dtype)
        off = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).cuda()
        kb.kroquant_cache_write(cache, x[0], x[1], table.cuda(), offsets=off)
    assert C >= d
    return cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")


def check(out, q, cache, table, lengths, scale, window=0, lse=None):
    n, q_heads, d = q.shape
    group = q_heads // cache.heads
    half_w = 2.0 ** -17 if cache.format == "16bit" and cache.dtype is torch.bfloat16 else 2.0 ** -11
    for i, length in enumerate(lengths.tolist()):
        length = max(0, min(length, table.shape[1] * cache.page_size))
        first = max(0, length - window) if window else 0
        k, v, live = cr.gather(cache, table[i], first, length)
        qs = q[i].double().view(cache.heads, group, d)
        if not bool(live.any()):
            assert bool((out[i] == 0).all())
            assert lse is None or bool((lse[i] == -math.inf).all())
            continue
        score = torch.where(live, scale * (qs @ k.mT), torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
        w = torch.softmax(score, -1)
        want = (w @ v).reshape(q_heads, d)
        size = (w @ v.abs()).reshape(q_heads, d)
        delta = (d / 16 + 8) * 2.0 ** -23 * abs(scale) * (qs.abs() @ k.abs().mT).amax(-1).reshape(q_heads, 1)
        least = 0 if half_w < 2.0 ** -11 else 2.0 ** -34 * 1.75 * (length - first) * v.abs().amax((1, 2)).repeat_interleave(group)[:, None]
        tol = least + (half_w + 2.0 ** -21 + 2 * delta + ((length - first) / 16 + 8) * 2.0 ** -23) * size
        tol = tol + torch.finfo(out.dtype).eps / 2 * (want.abs() + tol) + torch.finfo(out.dtype).smallest_normal
        over = (out[i].double() - want).abs() - tol
        assert bool((over <= 0).all()), (i, length, float(over.max()), float(size.max()))
        if lse is not None:
            exact = torch.logsumexp(score, -1).reshape(q_heads)
            # fp32 of the value, of the maximum in units of log 2, and the sum's relative error
            assert bool(((lse[i].double() - exact).abs() <= 2.0 ** -22 * (exact.abs() + 1) + delta[:, 0] + 2.0 ** -21 + (length / 16) * 2.0 ** -23).all())


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("d", [64, 128, 256, 1, 40, 72, 96, 112, 160, 200])
def test_head_widths(form, dtype, d):
    lengths = [1, 17, 300, 0, 129, 1000]
    cache, table, n = make(lengths, 2, d, 16, form, dtype, d)
    q = 1.5 * torch.randn(len(lengths), 6, d, device="cuda", generator=gen(1))
    out, lse = kb.kroquant_cache_attention(q.to(dtype), cache, table, n, lse=True, out_dtype=torch.float32)
    check(out, q.to(dtype), cache, table, n, d ** -0.5, lse=lse)
    assert torch.equal(kb.kroquant_cache_attention(q.to(dtype), cache, table, n), out.to(dtype))
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 9, 16, 17, 40])
def test_head_groups(form, dtype, group):
    lengths = [700, 33]
    cache, table, n = make(lengths, 3, 128, 8, form, dtype, group)
    q = torch.randn(2, 3 * group, 128, device="cuda", generator=gen(2)).to(dtype)
    out, lse = kb.kroquant_cache_attention(q, cache, table, n, lse=True, scale=0.2)
    check(out, q, cache, table, n, 0.2, lse=lse)


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("size", [1, 3, 16, 31, 32, 33, 64, 200, 5000])
@pytest.mark.parametrize("window", [0, 1, 50, 4096])
def test_pages_and_windows(form, dtype, size, window):
    lengths = [1, size, size + 1, 2 * size + 5, 4999, 0]
    cache, table, n = make(lengths, 1, 64, size, form, dtype, size, width=5000 // size + 3)
    q = torch.randn(len(lengths), 4, 64, device="cuda", generator=gen(3)).to(dtype)
    out, lse = kb.kroquant_cache_attention(q, cache, table, n, lse=True, window=window, out_dtype=torch.float32)
    check(out, q, cache, table, n, 0.125, window, lse)


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("heads,sequences", [(1, 1), (8, 1), (2, 9)])
def test_long_sequences_are_split_and_joined(form, dtype, heads, sequences):
    lengths = [20011 - 1999 * i for i in range(sequences)]
    cache, table, n = make(lengths, heads, 128, 64, form, dtype, heads)
    q = torch.randn(sequences, 4 * heads, 128, device="cuda", generator=gen(4)).to(dtype)
    out, lse = kb.kroquant_cache_attention(q, cache, table, n, lse=True, out_dtype=torch.float32)
    check(out, q, cache, table, n, 128 ** -0.5, lse=lse)
    for _ in range(3):                                                   # the same bits every time
        again = kb.kroquant_cache_attention(q, cache, table, n, lse=True, out_dtype=torch.float32)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("form,dtype", FORMATS)
def test_many_sequences(form, dtype):
    lengths = [(37 * i) % 611 if i % 5 else 0 for i in range(333)]
    cache, table, n = make(lengths, 2, 64, 16, form, dtype, 5)
    q = torch.randn(333, 2, 64, device="cuda", generator=gen(5)).to(dtype)
    check(kb.kroquant_cache_attention(q, cache, table, n), q, cache, table, n, 0.125)
    wide = torch.cat([table, torch.full((333, 3000), -1, dtype=torch.int32, device="cuda")], 1)      # room for more than the rows have
    check(kb.kroquant_cache_attention(q, cache, wide, n), q, cache, wide, n, 0.125)


@pytest.mark.parametrize("form,dtype", FORMATS)
def test_places_without_a_page_and_lengths_beyond_the_table(form, dtype):
    cache, table, n = make([100, 100, 100, 100, 64], 2, 64, 16, form, dtype, 6)
    table[0, 2], table[1, 0], table[2, 3] = -1, cache.pages, -2 ** 31
    table[3] = -1
    # a page the first sequence's positions fill only in part now counts to its end: zeros there
    n = torch.tensor([100, 96, 90, 100, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    q = torch.randn(5, 4, 64, device="cuda", generator=gen(6)).to(dtype)
    out, lse = kb.kroquant_cache_attention(q, cache, table, n, lse=True)
    check(out, q, cache, table, n, 0.125, lse=lse)
    out, lse = kb.kroquant_cache_attention(q, cache, table, torch.tensor([-1, -2 ** 31, 0, 5, 1], dtype=torch.int32, device="cuda"), lse=True)
    assert bool((out[:4] == 0).all()) and bool((lse[:4] == -math.inf).all()) and bool(torch.isfinite(lse[4]).all())
    out = kb.kroquant_cache_attention(q, cache, table[:, :0], n)
    assert bool((out == 0).all())


@pytest.mark.parametrize("form,dtype", FORMATS)
@pytest.mark.parametrize("gain,q_gain", [(1, 60.0), (2.0 ** -10, 1.0), (2.0 ** 7, 0.1), (1, 0.0), (1, 2.0 ** -12)])
def test_sizes_of_scores_and_values(form, dtype, gain, q_gain):
    """One position takes all, all positions weigh the same, very small and large keys and values."""
    cache, table, n = make([900, 40], 2, 128, 16, form, dtype, 7, gain=gain)
    q = (q_gain * torch.randn(2, 8, 128, device="cuda", generator=gen(7))).to(dtype)
    out, lse = kb.kroquant_cache_attention(q, cache, table, n, lse=True, out_dtype=torch.float32)
    check(out, q, cache, table, n, 128 ** -0.5, lse=lse)


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("where", [0, 5, 899])
def test_a_loud_position_does_not_cost_the_others_their_digits(form, where):
    """Values 2^12 times the others' at a position that hardly counts; keys of very unequal blocks."""
    cache, table, n = make([900], 1, 128, 16, form, torch.bfloat16, 8)
    x = torch.randn(1, 1, 128, device="cuda", generator=gen(8))
    k, v = (x * torch.exp2(torch.arange(128, device="cuda") // 32 * 6.0 - 12)).bfloat16(), (4096 * x).bfloat16()
    kb.kroquant_cache_write(cache, k, v, table, starts=torch.tensor([where], dtype=torch.int32, device="cuda"))
    q = torch.randn(1, 4, 128, device="cuda", generator=gen(9)).bfloat16()
    q[0, :2] = -(x[0, 0] * torch.exp2(6 - torch.arange(128, device="cuda") // 32 * 3.0)).bfloat16()
    out = kb.kroquant_cache_attention(q, cache, table, n, out_dtype=torch.float32)
    check(out, q, cache, table, n, 128 ** -0.5)


@pytest.mark.parametrize("form,dtype", FORMATS)
def test_strides_and_types(form, dtype):
    cache, table, n = make([50, 400, 3], 2, 80, 16, form, dtype, 10)
    packed = torch.randn(3, 11, 81, device="cuda", generator=gen(10)).to(dtype)
    q = packed[:, 1:7, 1:]                                               # odd addresses, gaps between heads
    wide = torch.cat([table, table], 1)[:, : table.shape[1]]             # rows with a pitch
    for t in (torch.float32, torch.bfloat16, torch.float16):
        room = torch.full((6, 3, 83), 7.0, dtype=t, device="cuda")
        out = room.transpose(0, 1)[:, :, 1:81]
        got = kb.kroquant_cache_attention(q, cache, wide, n, out=out)
        assert got is out
        check(out, q, cache, table, n, 80 ** -0.5)
        assert bool((room[..., 0] == 7).all()) and bool((room[..., 81:] == 7).all())


def test_not_finite_values():
    """NaN and infinity where nobody looks change nothing; a NaN key or value reaches the heads that see it and no others."""
    cache, table, n = make([40, 40], 2, 64, 16, "16bit", torch.bfloat16, 11)
    q = torch.randn(2, 4, 64, device="cuda", generator=gen(11)).bfloat16()
    want = kb.kroquant_cache_attention(q, cache, table, n)
    assert bool(torch.isfinite(want).all())                              # (unused cells are NaN throughout)
    cache.k[int(table[0, 2]), :, 8:] = float("inf")                      # positions 40 .. 47
    assert torch.equal(kb.kroquant_cache_attention(q, cache, table, n), want)
    cache.v[int(table[0, 0]), 1, 3, 5] = float("nan")
    got = kb.kroquant_cache_attention(q, cache, table, n)
    assert bool(torch.isnan(got[0, 2:, 5]).all())
    got[0, 2:, 5] = want[0, 2:, 5]
    assert torch.equal(got, want)
    cache.k[int(table[1, 1]), 0, 2, 0] = float("nan")
    got = kb.kroquant_cache_attention(q, cache, table, n)
    assert bool(torch.isnan(got[1, :2]).all()) and torch.equal(got[1, 2:], want[1, 2:])


def test_cache_beyond_32_bit_offsets():
    heads, d, size = 4, 128, 256
    row = heads * size * d * 2
    pages = (5 << 30) // row
    k, v = (torch.empty(pages, heads, size, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = kb.KVCache(k, v, head_dim=d, format="16bit")
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    x = torch.randn(2, 3 * size, heads, d, device="cuda", generator=gen(12)).bfloat16()
    kb.kroquant_cache_write(cache, x[0], x[1], table, offsets=torch.tensor([0, 3 * size], dtype=torch.int32, device="cuda"))
    q = torch.randn(1, 8, d, device="cuda", generator=gen(13)).bfloat16()
    n = torch.tensor([3 * size - 5], dtype=torch.int32, device="cuda")
    check(kb.kroquant_cache_attention(q, cache, table, n), q, cache, table, n, d ** -0.5)


def test_streams_and_graphs_share_nothing():
    """Two calls at once on two streams, and two captured calls replayed after the lengths and the cache have changed."""
    probs = [make([30000 - 7 * i, 500], 2, 128, 64, "mxfp8", torch.bfloat16, 20 + i) for i in range(2)]
    qs = [torch.randn(2, 8, 128, device="cuda", generator=gen(30 + i)).bfloat16() for i in range(2)]
    want = [kb.kroquant_cache_attention(q, *p) for q, p in zip(qs, probs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(5):
        for s, q, p, w in zip(streams, qs, probs, want):
            outs.append((kb.kroquant_cache_attention(q, *p, stream=s), w))
    torch.cuda.synchronize()
    for o, w in outs:
        assert torch.equal(o, w)
    graphs, got = [], []
    for q, p in zip(qs, probs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(kb.kroquant_cache_attention(q, *p))
    for _, _, n in probs:
        n.copy_(torch.tensor([123, 20000], device="cuda"))
        n[1] = 450
    want = [kb.kroquant_cache_attention(q, *p) for q, p in zip(qs, probs)]
    for s, gr in zip(streams, graphs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            gr.replay()
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        assert torch.equal(o, w)


def test_a_page_for_every_sequence_and_a_sequence_twice():
    """Sequences may read the same pages: rows of a batch that share a prefix, or all of it."""
    cache, table, n = make([3000], 2, 64, 16, "mxfp4", torch.bfloat16, 60)
    q = torch.randn(1, 8, 64, device="cuda", generator=gen(60)).bfloat16()
    one = kb.kroquant_cache_attention(q, cache, table, n, out_dtype=torch.float32)
    many = kb.kroquant_cache_attention(q.expand(40, 8, 64), cache, table.expand(40, table.shape[1]), n.repeat(40), out_dtype=torch.float32)
    for i in range(40):
        check(many[i : i + 1], q, cache, table, n, 0.125)
    check(one, q, cache, table, n, 0.125)


def test_scratch_is_as_large_as_it_says():
    import ctypes as C
    cache, table, n = make([9000], 2, 64, 16, "mxfp4", torch.bfloat16, 40)
    q = torch.randn(1, 4, 64, device="cuda", generator=gen(40)).bfloat16()
    want = kb.kroquant_cache_attention(q, cache, table, n)
    out, L = torch.zeros_like(want), kb.load_library()
    a = kb._AttentionArgs(1, 4, 1, 1, q.data_ptr(), out.data_ptr(), 256, 64, 256, 64, table.data_ptr(), table.stride(0), table.shape[1], n.data_ptr(), 0, 0.125, None)
    size = L.kroquant_cache_attention_scratch_bytes(cache._at, C.addressof(a))
    assert size > 0
    scratch = torch.full((size + 4096,), 77, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert L.kroquant_cache_attention(cache._at, C.addressof(a), scratch.data_ptr(), size - 1, stream) == 2
    assert L.kroquant_cache_attention(cache._at, C.addressof(a), None, size, stream) == 1
    assert L.kroquant_cache_attention(cache._at, C.addressof(a), scratch.data_ptr() + 8, size, stream) == 3
    assert L.kroquant_cache_attention(cache._at, C.addressof(a), scratch.data_ptr(), size, stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want) and bool((scratch[size:] == 77).all())


def test_refusals():
    c, table, n = make([5, 9], 2, 64, 8, "mxfp4", torch.bfloat16, 50)
    b, _, _ = make([5, 9], 2, 64, 8, "16bit", torch.float16, 50)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert kb.kroquant_cache_attention(q[:0], c, table[:0], n[:0]).shape == (0, 4, 64)
    for args, kw in (((q[:1], c, table, n), {}), ((q[:, :3], c, table, n), {}), ((q[:, :, :32], c, table, n), {}), ((q.float(), c, table, n), {}), ((q, b, table, n), {}),
                     ((q.cpu(), c, table, n), {}), ((q, c, table.cpu(), n), {}), ((q, c, table, n.long()), {}), ((q, c, table, n[:1]), {}), ((q, c, table, n.cpu()), {}),
                     ((q, c, table, n), dict(window=-1)), ((q, c, table, n), dict(out=q[:1])), ((q, c, table, n), dict(out_dtype=torch.int8)),
                     ((q, c, table, n), dict(out=q[:, :1].expand(2, 4, 64))), ((q, c, table, n), dict(out=q)), ((q.transpose(1, 2), c, table, n), {})):
        with pytest.raises(ValueError):
            kb.kroquant_cache_attention(*args, **kw)
