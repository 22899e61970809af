"""CPU-only: outputs of a decode step's calls that share memory with what the call reads, or with one another, are refused before any launch."""
import random

import pytest
import torch

from paper_2607_21446_b200 import binding as kb


def addresses(t):
    """Byte addresses of a CPU tensor's elements."""
    at = torch.zeros(t.shape, dtype=torch.int64)
    for i, (n, s) in enumerate(zip(t.shape, t.stride())):
        at += (torch.arange(n) * s * t.element_size()).view([-1 if k == i else 1 for k in range(t.dim())])
    return {t.data_ptr() + int(a) + b for a in at.flatten() for b in range(t.element_size())}


def test_meet_never_overlooks_a_shared_byte():
    rng = random.Random(1)
    room = torch.zeros(4096, dtype=torch.uint8)
    apart = 0
    for _ in range(3000):
        views = []
        for _ in range(2):
            t = room.view(rng.choice([torch.uint8, torch.bfloat16, torch.float32]))
            shape = [rng.randint(1, 4) for _ in range(rng.randint(1, 4))]
            stride = [rng.choice([0, 1, 2, 3, 4, 8, 12, 16, 24, 32, 48, 64]) for _ in shape]
            reach = sum((n - 1) * s for n, s in zip(shape, stride))
            views.append(t.as_strided(shape, stride, rng.randint(0, min(40, t.numel() - reach - 1))))
        met = bool(addresses(views[0]) & addresses(views[1]))
        assert kb._meet(*views) == kb._meet(*views[::-1])
        if not kb._meet(*views):
            apart += 1
            assert not met
    assert apart > 500


def test_parts_of_packed_rows_do_not_meet():
    packed = torch.zeros(5, 11, 8, dtype=torch.bfloat16)
    q, k, v = packed.split((6, 2, 3), 1)
    pairs = [(q, k), (q, v), (k, v), (q[..., :4], q[..., 4:]), (packed[::2], packed[1::2]), (packed[:0], packed), (q[:2], q[2:])]
    batched = torch.zeros(3, 5, 11, 8)
    pairs += [(batched[:, :, :6], batched[:, :, 6:]), (batched[:, :2], batched[:, 2:]), (batched[..., :3], batched[..., 3:])]
    pairs += [(packed[:, :10:2], packed[:, 1:11:2]), (packed[:, ::3, :5], packed[:, 1::3]), (batched[:, :, 4:9:2, 1:], batched[:, :, 1::2])]
    heads_first = batched.transpose(1, 2)
    pairs += [(heads_first[:, :6], heads_first[:, 6:]), (batched.expand(3, 5, 11, 8)[:1], batched[1:])]
    for a, b in pairs:
        assert not kb._meet(a, b) and not kb._meet(b, a)
    for a, b in ((q, q), (q, packed), (packed[:, 0:8], packed[:, 4:11]), (packed[:3], packed[2:]), (q, packed[:, 5:7]), (packed.view(5, 88), k)):
        assert kb._meet(a, b) and kb._meet(b, a)


@pytest.fixture
def here(monkeypatch):
    """CPU tensors pass for tensors on the current device: what the checks do not refuse reaches the library, which finds no device."""
    monkeypatch.setattr(kb, "_device", lambda: -1)


def refused(call, *args, **kw):
    with pytest.raises(ValueError):
        call(*args, **kw)


def passes(call, *args, **kw):
    if not torch.cuda.is_available():                                    # (on a device the call would run on these addresses)
        with pytest.raises(kb.KroQuantError):
            call(*args, **kw)


def test_few_row_product_refuses_out_on_x(here):
    M, N = 3, 64
    x = torch.zeros(M, N, dtype=torch.bfloat16)
    w, s = torch.zeros(N, N // 2, dtype=torch.uint8), torch.zeros(kb.tiled_scale_bytes(N, N), dtype=torch.uint8)
    room = torch.zeros(M, 2 * N, dtype=torch.bfloat16)
    for a, out in ((x, x), (room[:, :N], room[:, N // 2 : N // 2 + N]), (room[:, 1 : N + 1], room[:, :N]), (x, x.view(torch.float16))):
        refused(kb.kroquant_linear_w4a16, a, w, s, out=out, stream=0)
        refused(kb.kroquant_linear_w4a16, a, w, s, out=out, residual=out, stream=0)
    passes(kb.kroquant_linear_w4a16, room[:, :N], w, s, out=room[:, N:], stream=0)
    passes(kb.kroquant_linear_w4a16, x, w, s, out=room[:, N:], residual=room[:, N:], stream=0)


def cache_of(form, dtype=torch.bfloat16):
    return kb.KVCache.empty(4, 8, 2, 64, form, dtype, device="cpu"), torch.zeros(3, 2, dtype=torch.int32)


@pytest.mark.parametrize("form", ["16bit", "mxfp8"])
def test_cache_read_refuses_outputs_on_one_another(here, form):
    cache, table = cache_of(form)
    room = torch.zeros(3, 6, 64, dtype=torch.bfloat16)
    k, v = room[:, :2], room[:, 2:4]
    for out in ((k, k), (k, room[:, 1:3]), (room[:, :4:2], room[:, 2:4]), (k, k.view(torch.float16).view(torch.bfloat16))):
        refused(kb.kroquant_cache_read, cache, table, 3, out=out, stream=0)
    if form == "16bit":                                                  # pages read into other pages
        offsets = torch.tensor([0, 8], dtype=torch.int32)
        passes(kb.kroquant_cache_read, cache, table[:1], 8, out=(cache.k[3].transpose(0, 1), cache.v[3].transpose(0, 1)), offsets=offsets, stream=0)
    passes(kb.kroquant_cache_read, cache, table, 3, out=(k, v), stream=0)
    passes(kb.kroquant_cache_read, cache, table, 3, out=(room[:, ::2][:, :2], room[:, 1::2][:, :2]), stream=0)


def test_rotary_refuses_outputs_on_what_it_reads_or_writes(here):
    where, f = torch.zeros(5, dtype=torch.int32), torch.ones(4, dtype=torch.float64)
    packed = torch.zeros(5, 11, 8, dtype=torch.bfloat16)
    q, k = packed[:, :6], packed[:, 6:8]
    room = torch.zeros(5, 16, 8, dtype=torch.bfloat16)
    rot = lambda q, k, out, **kw: kb.kroquant_rotary(q, k, where, f, out=out, stream=0, **kw)  # noqa: E731
    for out in ((packed[:, 1:7], k), (room[:, :6], packed[:, 5:7]), (room[:, :6], room[:, 5:7]), (packed[:, 2:8], room[:, :2]), (q, packed[:, 5:7]),
                (room[:, :6], q[:, :2]), (room[:, :6], room[:, :2])):
        refused(rot, q, k, out)
    for t in (where, f):
        inside = torch.as_strided(t.view(torch.bfloat16), (1, 1, 8), (8, 8, 1))
        refused(kb.kroquant_rotary, room[:1, :1], None, where[:1], f, out=inside, stream=0)
    refused(rot, q, None, packed[:, 1:7])
    batched = packed.view(1, 5, 11, 8).expand(2, 5, 11, 8)
    refused(rot, batched[:, :, :6], None, batched[:, :, :6])             # the same elements twice
    for out in ((q, k), (q, room[:, :2]), (room[:, :6], k), (room[:, :6], room[:, 6:8]), (room[:, ::2][:, :6], room[:, 1::2][:, :2])):
        passes(rot, q, k, out)
    two = torch.zeros(2, 5, 11, 8)
    passes(rot, two[:, :, :6], two[:, :, 6:8], (two[:, :, :6], two[:, :, 6:8]))
    one = torch.zeros(1, 6, 8).as_strided((1, 6, 8), (999, 8, 1))
    passes(kb.kroquant_rotary, one, None, where[:1], f, out=one.as_strided((1, 6, 8), (48, 8, 1)), stream=0)


@pytest.mark.parametrize("form", ["16bit", "mxfp4"])
def test_attention_refuses_out_on_q_or_on_the_cache(here, form):
    cache, table = cache_of(form)
    n = torch.ones(3, dtype=torch.int32)
    room = torch.zeros(3, 9, 64, dtype=torch.bfloat16)
    q = room[:, :4]
    inside = cache.v.view(torch.bfloat16).view(-1)[: 3 * 4 * 64].view(3, 4, 64)
    for out in (q, room[:, 1:5], room[:, 3:7], room[:, :8:2], inside, q.view(torch.float16)):
        refused(kb.kroquant_cache_attention, q, cache, table, n, out=out, stream=0)
    passes(kb.kroquant_cache_attention, q, cache, table, n, out=room[:, 4:8], stream=0)
    passes(kb.kroquant_cache_attention, room[:, :8:2], cache, table, n, out=room[:, 1:8:2], stream=0)


def test_cache_whose_buffers_overlap_is_not_written(here):
    table, one = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    c = kb.KVCache.empty(4, 8, 2, 64, "mxfp8", device="cpu")
    b = kb.KVCache.empty(4, 8, 2, 64, "16bit", device="cpu")
    for shared in (kb.KVCache(b.k, b.k, head_dim=64, format="16bit"), kb.KVCache(c.k, c.k, c.k_scales, c.v_scales, head_dim=64, format="mxfp8"),
                   kb.KVCache(c.k, c.v, c.k_scales, c.k_scales, head_dim=64, format="mxfp8")):
        refused(kb.kroquant_cache_write, shared, one, one, table, stream=0)
        passes(kb.kroquant_cache_read, shared, table, 3, out=(one, one.clone()), stream=0)
    halves = torch.zeros(8, 2, 8, 64, dtype=torch.bfloat16)
    passes(kb.kroquant_cache_write, kb.KVCache(halves[:4], halves[4:], head_dim=64, format="16bit"), one, one, table, stream=0)
