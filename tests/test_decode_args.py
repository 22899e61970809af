"""CPU-only: what the entry points of a decode step refuse before any CUDA call, and what the cache handle refuses."""
import ctypes as C

import pytest
import torch

from paper_2607_21446_b200 import binding as kb

P = 4096                                     # a non-null, aligned address; nothing is launched


def struct(cls, base, kw):
    a = cls()
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def rotary(**kw):
    a = kb._RotaryArgs()
    kb.load_library().kroquant_rotary_args_default(C.addressof(a))
    for k, v in {**dict(dtype=1, tokens=4, head_dim=64, axis0=64, frequencies=P, positions=P, x0=P, out0=P, heads0=2), **kw}.items():
        setattr(a, k, v)
    return kb.load_library().kroquant_rotary(C.addressof(a), None)


def cache(**kw):
    return struct(kb._Cache, dict(format=2, dtype=1, pages=4, page_size=16, heads=2, head_dim=64, k=P, v=P, k_scales=P, v_scales=P), kw)


def rows(write=True, c=None, **kw):
    c = cache() if c is None else c
    r = struct(kb._CacheRows, dict(rows=2, sequences=2, table=P, table_stride=4, table_width=4, dtype=1, k=P, v=P), kw)
    fn = kb.load_library().kroquant_cache_write if write else kb.load_library().kroquant_cache_read
    return fn(C.addressof(c), C.addressof(r), None)


def attention(c=None, scratch=P, nbytes=1 << 40, **kw):
    c = cache() if c is None else c
    a = struct(kb._AttentionArgs, dict(sequences=2, q_heads=4, q_dtype=1, out_dtype=1, q=P, out=P, table=P, table_stride=4, table_width=4,
                                       lengths=P, scale=1.0), kw)
    return kb.load_library().kroquant_cache_attention(C.addressof(c), C.addressof(a), scratch, nbytes, None)


def w4a16(**kw):
    a = dict(x=P, xt=0, ld=64, b=P, s=P, M=2, N=64, K=64, e=None, out=P, dtype=1, ldo=64)
    a.update(kw)
    e = a["e"]
    return kb.load_library().kroquant_linear_w4a16(a["x"], a["xt"], a["ld"], a["b"], a["s"], a["M"], a["N"], a["K"],
                                                   None if e is None else C.addressof(e), a["out"], a["dtype"], a["ldo"], None)


def test_rotary_refusals():
    assert kb.load_library().kroquant_rotary(None, None) == 1
    assert rotary(frequencies=None) == 1 and rotary(positions=None) == 1 and rotary(x0=None) == 1 and rotary(out0=None) == 1
    assert rotary(x1=P, heads1=1) == 1 and rotary(out1=P, heads1=1) == 1
    assert rotary(head_dim=0) == 2 and rotary(head_dim=513) == 2 and rotary(tokens=-1) == 2 and rotary(heads0=0) == 2
    assert rotary(axes=0) == 2 and rotary(axes=5) == 2 and rotary(axis0=66) == 2 and rotary(axis0=33) == 2 and rotary(axis0=0) == 2
    assert rotary(axes=2, axis0=32, axis1=34) == 2 and rotary(axis0=-2) == 2 and rotary(batches=1 << 20, tokens=1 << 20) == 2
    assert rotary(x1=P, out1=P, heads1=0) == 2
    assert rotary(x0=P + 1) == 3 and rotary(out0=P + 1) == 3 and rotary(frequencies=P + 4) == 3 and rotary(positions=P + 2) == 3
    assert rotary(dtype=0, x0=P + 2) == 3
    assert rotary(dtype=3) == 5 and rotary(layout=2) == 5 and rotary(inverse=2) == 5 and rotary(positions_f32=7) == 5
    assert rotary(tokens=0, x0=None) == 0 and rotary(batches=0, frequencies=None) == 0


@pytest.mark.parametrize("write", [True, False])
def test_cache_refusals(write):
    L = kb.load_library()
    fn = L.kroquant_cache_write if write else L.kroquant_cache_read
    assert fn(None, P, None) == 1 and fn(P, None, None) == 1
    for bad in (dict(k=None), dict(v=None), dict(k_scales=None)):
        assert rows(write, cache(**bad)) == 1
    assert rows(write, k=None) == 1 and rows(write, table=None) == 1
    for bad in (dict(pages=0), dict(page_size=0), dict(heads=0), dict(head_dim=0), dict(head_dim=257), dict(pages=1 << 28)):
        assert rows(write, cache(**bad)) == 2
    assert rows(write, rows=-1) == 2 and rows(write, sequences=-1) == 2 and rows(write, rows=3) == 2 and rows(write, table_width=-1) == 2
    assert rows(write, rows=1 << 31, offsets=P) == 2
    assert rows(write, cache(k=P + 8)) == 3 and rows(write, cache(v_scales=P + 4)) == 3 and rows(write, k=P + 1) == 3 and rows(write, starts=P + 2) == 3
    assert rows(write, cache(format=3)) == 5 and rows(write, cache(format=0, dtype=0)) == 5 and rows(write, dtype=4) == 5
    if write:
        assert rows(write, dtype=0) == 5 and rows(write, cache(format=0, dtype=2), dtype=1) == 5
    assert rows(write, rows=0, sequences=0, k=None, table=None) == 0 and rows(write, rows=0, offsets=P, k=None) == 0
    assert rows(write, cache(k_scales=None, v_scales=None, format=0), rows=0, sequences=0) == 0


def test_attention_refusals():
    L = kb.load_library()
    assert L.kroquant_cache_attention(None, P, P, 0, None) == 1 and L.kroquant_cache_attention(P, None, P, 0, None) == 1
    assert attention(q=None) == 1 and attention(out=None) == 1 and attention(lengths=None) == 1 and attention(table=None) == 1
    assert attention(cache(k=None)) == 1
    assert attention(q_heads=0) == 2 and attention(q_heads=3) == 2 and attention(sequences=-1) == 2 and attention(window=-1) == 2
    assert attention(table_width=-1) == 2 and attention(table_width=1 << 27) == 2 and attention(cache(head_dim=300)) == 2
    assert attention(q=P + 1) == 3 and attention(out_dtype=0, out=P + 2) == 3 and attention(lengths=P + 2) == 3 and attention(lse=P + 1) == 3
    assert attention(cache(v=P + 8)) == 3
    assert attention(q_dtype=0) == 5 and attention(out_dtype=3) == 5 and attention(cache(format=0, dtype=2)) == 5
    assert attention(sequences=0, q=None) == 0
    assert L.kroquant_cache_attention_scratch_bytes(None, None) == 0


def test_w4a16_refusals():
    assert w4a16(x=None) == 1 and w4a16(b=None) == 1 and w4a16(s=None) == 1 and w4a16(out=None) == 1
    assert w4a16(M=-1) == 2 and w4a16(M=65) == 2 and w4a16(N=0) == 2 and w4a16(K=48) == 2 and w4a16(ld=63) == 2 and w4a16(ldo=63) == 2
    assert w4a16(x=P + 1) == 3 and w4a16(b=P + 8) == 3 and w4a16(s=P + 4) == 3 and w4a16(out=P + 1) == 3
    assert w4a16(xt=2) == 5 and w4a16(dtype=3) == 5
    e = kb._Epilogue()
    kb.load_library().kroquant_epilogue_default(C.addressof(e))
    e.activation = 9
    assert w4a16(e=e) == 5
    assert w4a16(M=0, x=None, out=None) == 0


def test_cache_handle():
    c = kb.KVCache.empty(3, 5, 2, 72, "mxfp4", device="cpu")
    assert c.k.shape == (3, 2, 5, 48) and c.k_scales.shape == (3, 2, 5, 4) and c.dtype is torch.bfloat16
    assert kb.KVCache.empty(3, 5, 2, 129, "mxfp8", device="cpu").v_scales.shape == (3, 2, 5, 8)
    b = kb.KVCache.empty(1, 1, 1, 1, "16bit", torch.float16, device="cpu")
    assert b.k.shape == (1, 1, 1, 32) and b.dtype is torch.float16 and b.k_scales is None
    for bad in (dict(head_dim=257), dict(format="fp8"), dict(head_dim=128), dict(dtype=torch.float32)):
        with pytest.raises(ValueError):
            kb.KVCache(c.k, c.v, c.k_scales, c.v_scales, **{**dict(head_dim=72, format="mxfp4"), **bad})
    for bufs in ((c.k, c.v), (c.k, c.v, c.k_scales, c.v_scales[..., :3]), (c.k, c.v[:2], c.k_scales, c.v_scales),
                 (c.k.transpose(0, 1), c.v.transpose(0, 1), c.k_scales, c.v_scales), (c.k.char(), c.v.char(), c.k_scales, c.v_scales)):
        with pytest.raises(ValueError):
            kb.KVCache(*bufs, head_dim=72)
    with pytest.raises(ValueError):
        kb.KVCache(b.k, b.v, head_dim=1, format="16bit", dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kb.KVCache.empty(1, 1, 1, 64, "other", device="cpu")


def test_elements_apart_and_spans():
    t = torch.zeros(4, 6, 8)
    assert kb._apart(t) and kb._apart(t.transpose(0, 1)) and kb._apart(t[:, ::2, 2:5]) and kb._apart(t[:0])
    assert not kb._apart(t[:, :1].expand(4, 3, 8)) and not kb._apart(torch.zeros(30).as_strided((4, 3, 8), (2, 4, 1)))
    a, b = kb._span(t[1:3])
    assert a == t.data_ptr() + 4 * 48 and b == t.data_ptr() + 4 * 144


def test_frequencies():
    f = kb.rotary_frequencies((4, 6), theta=100.0, device="cpu")
    assert f.dtype is torch.float64 and torch.allclose(f, torch.tensor([1, 0.1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)], dtype=torch.float64), rtol=1e-15)


def test_packed_structs_have_the_layout_of_the_c_ones():
    import struct
    for pack, cls in ((kb._PACK_ROTARY, kb._RotaryArgs), (kb._PACK_ROWS, kb._CacheRows), (kb._PACK_ATTENTION, kb._AttentionArgs)):
        values = [i + 1 for i in range(len(cls._fields_))]
        a = cls.from_buffer_copy(pack(*values))
        assert [getattr(a, f[0]) for f in cls._fields_] == values
    assert struct.calcsize("@P") == 8
