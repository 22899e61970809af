"""What a kernel writes is what the next one in the stream reads, although that one may begin early: chains of calls captured into one graph, over
inputs that change from link to link, against the same calls one at a time.  Equal bits."""
import pytest
import torch

from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def same_in_one_graph(links, call):
    """call(i) -> tensors; each link once with a wait in front and behind, then all of them in one graph, three times."""
    want = []
    for i in range(links):
        torch.cuda.synchronize()
        want.append([t.clone() for t in call(i)])
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [call(i) for i in range(links)]
    for _ in range(3):
        for link in got:
            for t in link:
                t.view(torch.uint8).fill_(0x7F)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b))
    assert kb.kroquant_last_device_error() == 0


@pytest.mark.parametrize("form", ["16bit", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("d,layout", [(128, "half"), (72, "half"), (64, "interleaved")])
def test_rotary_in_place_then_write_then_read(form, d, layout):
    rows, heads, size = 700, 6, 16
    x = torch.randn(8, rows, 3 * heads, d, device="cuda", generator=gen(d)).bfloat16()
    cache = kb.KVCache.empty(rows // size + 1, size, heads, d, form)
    table = torch.arange(rows // size + 1, dtype=torch.int32, device="cuda")[None]
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    where, f = torch.arange(rows, dtype=torch.int32, device="cuda"), kb.rotary_frequencies([d])
    packed = torch.empty_like(x[0])

    def link(i):
        packed.copy_(x[i])
        q, k, v = packed.split(heads, 1)
        kb.kroquant_rotary(q, k, where, f, layout=layout, out=(q, k))
        kb.kroquant_cache_write(cache, k, v, table, offsets=offsets)
        return kb.kroquant_cache_read(cache, table, rows, offsets=offsets)

    same_in_one_graph(8, link)


def weight(rows, K, g):
    w = (torch.randn(rows, K, device="cuda", generator=g) * K ** -0.5).bfloat16()
    return kb.kroquant_mxfp4_quantize(w, scale_layout="tiled")


@pytest.mark.parametrize("M", [8, 300])
def test_row_scales_from_the_product_before(M):
    """A product of few rows with one column as router weights of the next product."""
    g = gen(M)
    K, N = 1152, 640
    x = torch.randn(8, M, K, device="cuda", generator=g).bfloat16()
    router, w = weight(1, K, g), weight(N, K, g)
    scales = torch.empty(M, 1, device="cuda")

    def link(i):
        a = kb.kroquant_mxfp4_quantize(x[i], scale_layout="tiled") if M > 64 else None
        for r in range(0, M, 64):
            kb.kroquant_linear_w4a16(x[i, r : r + 64], *router, out=scales[r : r + 64])
        if M > 64:
            return (kb.kroquant_linear_mxfp4(*a, *w, row_scale=scales.view(-1)),)
        return (kb.kroquant_linear_w4a16(x[i], *w, row_scale=scales.view(-1)),)

    same_in_one_graph(8, link)


@pytest.mark.parametrize("rows,d,dtype", [(64, 1152, torch.float32), (3000, 1152, torch.bfloat16), (700, 5600, torch.float32), (90, 203, torch.float16)])
def test_norm_vectors_from_the_product_before(rows, d, dtype):
    """The modulation layer's product of one row gives gate, scale and shift of the norm behind it; then the norm's backward pass."""
    g = gen(d)
    K, D = 256, (d + 7) // 8 * 8
    w = weight(3 * D, K, g)
    t = torch.randn(8, 1, K, device="cuda", generator=g).bfloat16()
    x, y, dn = (torch.randn(rows, d, device="cuda", generator=g).bfloat16() for _ in range(3))
    six = torch.empty(1, 3 * D, dtype=dtype, device="cuda")

    def link(i):
        kb.kroquant_linear_w4a16(t[i], *w, out=six)
        gate, scale, shift = (six[:, j * D : j * D + d] for j in range(3))
        h, n = kb.kroquant_norm_residual(x, y, gate=gate, scale=scale, shift=shift, norm="layer")
        kb.kroquant_linear_w4a16(t[i], *w, out=six)
        back = kb.kroquant_norm_residual_grad(dn, h, y=y, gate=gate, scale=scale, shift=shift, norm="layer")
        return h, n, back["dx"], back["dy"], back["dscale"]

    same_in_one_graph(8, link)


@pytest.mark.parametrize("tokens,d", [(300, 1152), (2, 4608), (1, 40960)])
@pytest.mark.parametrize("staged", [True, False])
def test_scale_vector_from_the_product_before(tokens, d, staged):
    g = gen(d)
    w = weight(d, 256, g)
    t = torch.randn(8, 1, 256, device="cuda", generator=g).bfloat16()
    x = torch.randn(tokens, d, device="cuda", generator=g).bfloat16()
    s = torch.empty(1, d, device="cuda")
    tuning = None if staged else kb.Tuning(compare_staged=0)

    def link(i):
        kb.kroquant_linear_w4a16(t[i], *w, out=s)
        return kb.kroquant_scale_quantize(x, s.view(-1), tuning=tuning)

    same_in_one_graph(8, link)
