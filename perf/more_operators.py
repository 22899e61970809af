"""Operators of a quantized transformer that takes one step at a time: cases, inputs, plain forms, 64-bit values.

Four operators, which a block with MXFP4 weights runs for its new tokens:

* ``rotary``    rotary positions with one to four axes (time, height, width, ...) on queries and keys in one pass:
                (a, b) -> (a cos t - b sin t, a sin t + b cos t) with t = position[axis of the pair] * frequency[pair], and the
                backward pass, which turns the gradients by -t;
* ``store``     new keys and values written to a paged cache in MXFP8 or MXFP4 (or as they are), then the whole context read
                back in 16 bits, as a step over a chunk of tokens does;
* ``attention`` one new token of every sequence over its pages of the cache: softmax(scale q K^T) V, grouped heads, optionally
                only the last `window` positions;
* ``product``   out = r * residual + act(x W^T + bias) for a few rows of x in 16 bits and W in MXFP4.

The cache: pages of `page_size` positions, [pages][heads][page_size][row], a row being the head's channels filled up with zeros
to a multiple of 32; 16-bit values, E4M3 codes or packed E2M1 codes, and for the codes one E8M0 byte per 32 channels in rows of
a multiple of four bytes.  A table gives the pages of each sequence in order.

The plain form (``own`` false) is elementary torch arithmetic in 32 bits with one rounding at the end (angles in 64);
``exact`` computes the same definitions in 64 bits and is written separately.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
CODE_BITS = {"16bit": 16, "mxfp8": 8, "mxfp4": 4}

_package = None


def _binding():
    global _package
    if _package is None:
        from paper_2607_21446_b200 import binding
        _package = binding
    return _package


# ---------------------------------------------------------------------------------------------------------------- cases
def _rotary(name, tokens, heads, kv_heads, dim, axes, layout="interleaved", inverse=False, far=0, dtype="bf16"):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "axes": "x".join(map(str, axes)), "layout": layout, "inverse": inverse, "far": far, "dtype": dtype}


def _store(name, sequences, history, new, kv_heads, dim, page_size, form, dtype="bf16"):
    return {"name": name, "op": "store", "sequences": sequences, "history": history, "new": new, "kv_heads": kv_heads, "dim": dim,
            "page_size": page_size, "format": form, "dtype": dtype}


def _attention(name, sequences, length, heads, kv_heads, dim, page_size, form, spread="even", window=0, dtype="bf16"):
    return {"name": name, "op": "attention", "sequences": sequences, "length": length, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "page_size": page_size, "format": form, "spread": spread, "window": window, "dtype": dtype}


def _product(name, M, N, K, act="none", glu=False, bias=False, residual=False, dtype="bf16", out="bf16"):
    return {"name": name, "op": "product", "M": M, "N": N, "K": K, "act": act, "glu": glu, "bias": bias, "residual": residual,
            "dtype": dtype, "out": out}


def listed():
    return [
        # a decode step's token far into a long sequence, grouped heads: latency
        _rotary("rotary_one_token", 1, 32, 8, 128, (128,), layout="half", far=1000000),
        # text and image tokens of a 4608-wide block, three axes (text index, height, width)
        _rotary("rotary_image", 4608, 36, 36, 128, (16, 56, 56)),
        # backward over a clip's tokens (time, height, width) of a 1152-wide block, a head width that is no multiple of 16
        _rotary("rotary_video_grad", 10007, 16, 16, 72, (24, 24, 24), layout="half", inverse=True, dtype="f16"),
        # a short prompt continued by a few tokens
        _store("store_small", 1, 283, 17, 8, 128, 16, "mxfp8"),
        # chunks of four long sequences, 4-bit cache
        _store("store_chunk", 4, 12000, 1027, 8, 128, 16, "mxfp4"),
        # one short sequence in a 16-bit cache: latency
        _attention("attention_short", 1, 300, 32, 8, 128, 16, "16bit"),
        # a decode batch of unequal lengths, 8-bit cache
        _attention("attention_batch", 24, 8192, 32, 8, 128, 64, "mxfp8", spread="ragged"),
        # one very long sequence, 4-bit cache
        _attention("attention_long", 1, 131071, 32, 8, 128, 16, "mxfp4"),
        # a rolling window over frames in a 2240-wide block, every head with its own keys, an odd page size
        _attention("attention_window", 5, 9000, 20, 20, 112, 49, "16bit", window=4096, dtype="f16"),
        # the modulation layer of a 1152-wide block: one conditioning row, not quantized, six vectors out
        _product("modulation_row", 1, 6912, 1152, bias=True, dtype="f16", out="f32"),
        # a decode step of five sequences into the gated hidden layer
        _product("gated_decode", 5, 5632, 4096, act="silu", glu=True),
        # sixteen rows through the widest feed-forward product back into the residual stream
        _product("wide_16_rows", 16, 4608, 12288, bias=True, residual=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op, dtype = rng.choice(["rotary", "store", "attention", "attention", "product"]), rng.choice(["bf16", "f16"])
    if op == "product":
        while True:
            M, N, K = _log(rng, 1, 32), _log(rng, 32, 12288), 32 * _log(rng, 4, 384)
            glu = rng.random() < 0.4
            if N * (2 if glu else 1) * K <= 4608 * 12288:
                break
        case = _product("", M, N, K, rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), glu, rng.random() < 0.5,
                        rng.random() < 0.5, dtype, rng.choice(["bf16", "f16", "f32"]))
    elif op == "rotary":
        while True:
            dim = rng.choice([64, 72, 80, 96, 112, 128, 128, 256])
            kv_heads = _log(rng, 1, 32)
            heads = kv_heads * rng.choice([1, 1, 2, 4, 8])
            tokens = _log(rng, 1, 30000)
            if tokens * (heads + kv_heads) * dim <= 4608 * 72 * 128 and heads <= 64:
                break
        count, rest, axes = rng.choice([1, 2, 3, 3]), dim, []
        if rng.random() < 0.2:
            rest = dim // 4 * 2                                          # the other channels are not turned
        for i in range(count - 1):
            axes.append(2 * rng.randint(1, max(1, rest // 2 - (count - 1 - i)) // 2 + 1))
            rest -= axes[-1]
        axes.append(rest)
        case = _rotary("", tokens, heads, kv_heads, dim, axes, rng.choice(["interleaved", "half"]), rng.random() < 0.4,
                       rng.choice([0, 0, 100000, 2000000]), rng.choice(["bf16", "f16", "f32"]))
    else:
        kv_heads, dim = _log(rng, 1, 32), rng.choice([64, 72, 80, 96, 112, 128, 128, 256])
        form, page_size = rng.choice(["mxfp8", "mxfp4", "mxfp4", "16bit"]), rng.choice([1, 7, 16, 16, 32, 49, 64, 256])
        if op == "store":
            while True:
                sequences, history, new = _log(rng, 1, 64), _log(rng, 1, 30000), _log(rng, 1, 8192)
                if sequences * (history + new) * kv_heads * dim <= 4 * 13027 * 8 * 128:
                    break
            case = _store("", sequences, history - (history == 1), new, kv_heads, dim, page_size, form, dtype)
        else:
            while True:
                sequences, length = _log(rng, 1, 256), _log(rng, 1, 131071)
                if sequences * length * kv_heads * dim * CODE_BITS[form] <= 24 * 8192 * 8 * 128 * 8:
                    break
            heads = kv_heads * rng.choice([1, 2, 4, 4, 7, 8, 16])
            while heads > 128:
                heads -= kv_heads
            window = _log(rng, 1, 8192) if rng.random() < 0.25 else 0
            case = _attention("", sequences, length, heads, kv_heads, dim, page_size, form, rng.choice(["even", "ragged", "ragged"]),
                              window, dtype)
    del case["name"]
    return case


def _axes(case):
    return [int(a) for a in case["axes"].split("x")]


def _lengths(case):
    """Positions of every sequence.  Ragged: from the full length down; every seventh place of a padded batch is empty."""
    n, most = case["sequences"], case["length"]
    if case["spread"] == "even" or n == 1:
        return [most] * n
    return [0 if i % 7 == 6 else max(1, most * ((5 * i) % n + 1) // n) for i in range(n)]


def _chunks(case):
    """(positions already in the cache, new ones) of every sequence."""
    n = case["sequences"]
    return [(case["history"] * (n - i) // n, max(1, case["new"] * (i % 3 + 2) // 4) if n > 1 else case["new"]) for i in range(n)]


def _weight_rows(case):
    """Rows of the stored weight: a gated activation interleaves 32 gate rows with 32 value rows."""
    return 64 * ((case["N"] + 31) // 32) if case["glu"] else case["N"]


def _row_bytes(case):
    """Bytes of a head's keys at one position that carry something: codes and scales."""
    return case["dim"] * CODE_BITS[case["format"]] / 8 + (0 if case["format"] == "16bit" else (case["dim"] + 31) // 32)


def work(case):
    op = case["op"]
    if op == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2.0 * n * SIZES[case["dtype"]] + 4 * case["tokens"] * len(_axes(case)), "flops": 3.0 * n}
    if op == "store":
        new, total = sum(c for _, c in _chunks(case)), sum(h + c for h, c in _chunks(case))
        row = case["dim"] * SIZES[case["dtype"]]
        nbytes = 2 * case["kv_heads"] * (new * (row + _row_bytes(case)) + total * (row + _row_bytes(case)))
        return {"bytes": nbytes, "flops": 6.0 * case["kv_heads"] * case["dim"] * (new + total)}
    if op == "attention":
        seen = sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))
        nbytes = 2 * seen * case["kv_heads"] * _row_bytes(case) + 2 * case["sequences"] * case["heads"] * case["dim"] * SIZES[case["dtype"]]
        return {"bytes": nbytes, "flops": 4.0 * seen * case["heads"] * case["dim"]}
    M, N, K, R = case["M"], case["N"], case["K"], _weight_rows(case)
    nbytes = R * K * (0.5 + 1 / 32) + M * K * 2 + M * N * SIZES[case["out"]] * (2 if case["residual"] else 1) + 4 * R * case["bias"]
    return {"bytes": nbytes, "flops": 2.0 * M * R * K}


# --------------------------------------------------------------------------------------------------------------- inputs
def _steps(v, low, mantissa, top):
    """v float -> the nearest value of a small float format (ties to the even one): exponents from `low`, `mantissa` bits, <= top."""
    exponent = torch.frexp(v.abs())[1] - 1
    step = torch.ldexp(torch.ones_like(v), exponent.clamp_min(low) - mantissa)
    return (torch.round(v / step) * step).clamp(-top, top)


def _quantize(x, form):
    """float [..., 32 b] -> (values on the format's grid [..., 32 b], E8M0 bytes [..., b]): x ~ values * 2^(byte - 127)."""
    blocks = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    amax = blocks.abs().amax(-1)
    byte = (torch.frexp(amax)[1] - 1 - (8 if form == "mxfp8" else 2) + 127).clamp(0, 254)
    byte = torch.where(amax > 0, byte, torch.zeros_like(byte))
    scaled = torch.ldexp(blocks, (127 - byte)[..., None])
    grid = _steps(scaled, -6, 3, 448.0) if form == "mxfp8" else _steps(scaled, 0, 1, 6.0)
    return grid.reshape(x.shape), byte


def _codes(grid, form):
    """Values on the grid -> uint8 codes, packed in pairs (the even channel in the low half) for E2M1."""
    if form == "mxfp8":
        return grid.to(torch.float8_e4m3fn).view(torch.uint8)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=grid.device)
    code = torch.bucketize(grid.abs(), edges).to(torch.uint8) | (torch.signbit(grid).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _tile(scales):
    """E8M0 bytes [R, K/32] -> the 128 x 4 tiled layout, flat."""
    R, B = scales.shape
    rt, kt = (R + 127) // 128, (B + 3) // 4
    full = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=scales.device)
    full[:R, :B] = scales
    return full.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _fill_pages(state, case, pages, g):
    """Keys and values of every position of `pages` pages, encoded: a context as it lies in the cache before the step."""
    heads, size, dim, form = case["kv_heads"], case["page_size"], case["dim"], case["format"]
    padded = (dim + 31) // 32 * 32
    loud = torch.ones(heads, 1, dim, device="cuda")
    loud[:, :, torch.randint(0, dim, (max(1, dim // 40),), device="cuda", generator=g)] = 6.0
    for name, gain in (("k", loud), ("v", 0.5)):
        if form == "16bit":
            store = torch.zeros(pages, heads, size, padded, dtype=DTYPES[case["dtype"]], device="cuda")
        else:
            store = torch.zeros(pages, heads, size, padded * CODE_BITS[form] // 8, dtype=torch.uint8, device="cuda")
            scales = torch.zeros(pages, heads, size, (padded // 32 + 3) // 4 * 4, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 25) // (heads * size * padded))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = torch.zeros(n, heads, size, padded, device="cuda")
            x[..., :dim] = torch.randn(n, heads, size, dim, device="cuda", generator=g) * gain
            if form == "16bit":
                store[p : p + n] = x.to(store.dtype)
            else:
                grid, byte = _quantize(x, form)
                store[p : p + n] = _codes(grid, form)
                scales[p : p + n, :, :, : padded // 32] = byte.to(torch.uint8)
        state[name] = store
        state[name + "_scales"] = None if form == "16bit" else scales


def _paged(state, case, lengths, seed, g):
    """The cache and the table of a batch: pages in no particular order, unused entries -1."""
    size = case["page_size"]
    need = [(n + size - 1) // size for n in lengths]
    pages = max(1, sum(need))
    _fill_pages(state, case, pages, g)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed)))
    table, at = torch.full((len(lengths), max(1, max(need))), -1, dtype=torch.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = order[at : at + n].to(torch.int32)
        at += n
    state["table"] = table.cuda()
    if own:
        state["cache"] = _binding().KVCache(state["k"], state["v"], state["k_scales"], state["v_scales"], head_dim=case["dim"],
                                            format=case["format"])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    state, op = dict(case), case["op"]

    def normal(dtype, *shape, gain=1.0):
        return (gain * torch.randn(*shape, device="cuda", generator=g)).to(DTYPES[dtype])

    if op == "rotary":
        tokens, axes = case["tokens"], _axes(case)
        gain = 0.1 if case["inverse"] else 1.0
        state["q"] = normal(case["dtype"], tokens, case["heads"], case["dim"], gain=gain)
        state["k"] = normal(case["dtype"], tokens, case["kv_heads"], case["dim"], gain=gain)
        position, t = torch.zeros(tokens, len(axes), dtype=torch.int64), torch.arange(tokens)
        side = max(1, int(math.sqrt(min(tokens, 4096))))
        if len(axes) == 1:
            position[:, 0] = t
        else:                                                            # the last axes are places in a picture, the first counts pictures
            position[:, -1], position[:, -2] = t % side, t // side % side
            if len(axes) > 2:
                position[:, 0] = t // (side * side)
        position[:, 0] += case["far"] + int(seed) % 97
        state["positions"] = position.to(torch.int32).cuda()
        state["frequencies"] = torch.cat([10000.0 ** (-torch.arange(0, a, 2, dtype=torch.float64) / a) for a in axes]).cuda()
        return state
    if op == "store":
        chunks = _chunks(case)
        _paged(state, case, [h + n for h, n in chunks], seed, g)
        new = sum(n for _, n in chunks)
        state["k_new"] = normal(case["dtype"], new, case["kv_heads"], case["dim"])
        state["v_new"] = normal(case["dtype"], new, case["kv_heads"], case["dim"], gain=0.5)
        ends = [0], [0]
        for h, n in chunks:
            ends[0].append(ends[0][-1] + n)
            ends[1].append(ends[1][-1] + h + n)
        state["new_offsets"], state["all_offsets"] = (torch.tensor(e, dtype=torch.int32, device="cuda") for e in ends)
        state["starts"] = torch.tensor([h for h, _ in chunks], dtype=torch.int32, device="cuda")
        state["total"] = ends[1][-1]
        return state
    if op == "attention":
        lengths = _lengths(case)
        _paged(state, case, lengths, seed, g)
        state["q"] = normal(case["dtype"], case["sequences"], case["heads"], case["dim"], gain=1.5)
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        state["scale"] = case["dim"] ** -0.5
        return state
    M, N, K, R = case["M"], case["N"], case["K"], _weight_rows(case)
    x = torch.randn(M, K, device="cuda", generator=g)
    x[:, torch.randint(0, K, (max(1, K // 100),), device="cuda", generator=g)] *= 20.0
    state["x"] = x.to(DTYPES[case["dtype"]])
    grid, byte = _quantize(torch.randn(R, K, device="cuda", generator=g) / math.sqrt(K), "mxfp4")
    state["w_codes"], state["w_scales"] = _codes(grid, "mxfp4"), _tile(byte.to(torch.uint8))
    state["bias"] = 0.2 * torch.randn(R, device="cuda", generator=g) if case["bias"] else None
    state["residual"] = normal(case["out"], M, N) if case["residual"] else None
    return state


# ----------------------------------------------------------------------------------------------------------- plain form
def _pair_channels(case, device):
    """Channels of the first and second members of the turned pairs."""
    pairs = sum(_axes(case)) // 2
    p = torch.arange(pairs, device=device)
    return (2 * p, 2 * p + 1) if case["layout"] == "interleaved" else (p, p + pairs)


def _plain_rotary(s):
    axis = torch.cat([torch.full((a // 2,), i) for i, a in enumerate(_axes(s))]).to(s["q"].device)
    angle = s["positions"].double()[:, axis] * s["frequencies"]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if s["inverse"]:
        sin = -sin
    first, second = _pair_channels(s, s["q"].device)
    out = []
    for x in (s["q"], s["k"]):
        y = x.float()
        a, b = y[..., first], y[..., second]
        y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
        out.append(y.to(x.dtype))
    return tuple(out)


def _grid_values(form, device):
    """The value of every code: [16] of E2M1 or [256] of E4M3 (its two NaN codes as they are)."""
    if form == "mxfp8":
        return torch.arange(256, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn).float()
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=device)
    return torch.cat([grid, -grid])


def _decoded(codes, scales, form, dim):
    """Rows of the cache -> float values [..., dim]."""
    if form == "16bit":
        return codes[..., :dim].float()
    grid = _grid_values(form, codes.device)
    if form == "mxfp4":
        pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)        # byte -> (low code, high code)
        values = pairs[codes.int()].flatten(-2)
    else:
        values = grid[codes.int()]
    blocks = values.reshape(*values.shape[:-1], -1, 32)
    step = torch.exp2(scales[..., : blocks.shape[-2]].float() - 127)
    return (blocks * step[..., None]).flatten(-2)[..., :dim]


def _places(s, offsets, starts, rows):
    """Sequence and position of every packed row."""
    row = torch.arange(rows, device=offsets.device)
    which = (row[:, None] >= offsets[None, 1:]).sum(1)
    return which, row - offsets[which] + (0 if starts is None else starts[which])


def _plain_store(s):
    form, dim, size, dtype = s["format"], s["dim"], s["page_size"], DTYPES[s["dtype"]]
    padded = (dim + 31) // 32 * 32
    which, place = _places(s, s["new_offsets"], s["starts"], s["k_new"].shape[0])
    page, slot = s["table"][which, place // size].long(), place % size
    for name in ("k", "v"):
        x = s[name + "_new"]
        if form == "16bit":
            s[name][page, :, slot, :dim] = x
        else:
            wide = torch.zeros(*x.shape[:-1], padded, device=x.device)
            wide[..., :dim] = x.float()
            grid, byte = _quantize(wide, form)
            s[name][page, :, slot] = _codes(grid, form)
            s[name + "_scales"][page, :, slot, : padded // 32] = byte.to(torch.uint8)
    which, place = _places(s, s["all_offsets"], None, s["total"])
    page, slot = s["table"][which, place // size].long(), place % size
    out = []
    for name in ("k", "v"):
        scales = s[name + "_scales"]
        out.append(_decoded(s[name][page, :, slot], None if scales is None else scales[page, :, slot], form, dim).to(dtype))
    return tuple(out)


def _plain_attention(s):
    B, H, dim, size = s["sequences"], s["kv_heads"], s["dim"], s["page_size"]
    group, width = s["heads"] // H, s["table"].shape[1]
    out = torch.zeros(B, s["heads"], dim, device="cuda")
    for b in range(B):
        page = s["table"][b].clamp_min(0).long()
        keys, values = (_decoded(s[n][page], None if s[n + "_scales"] is None else s[n + "_scales"][page], s["format"], dim)
                        .transpose(0, 1).reshape(H, width * size, dim) for n in ("k", "v"))
        place, length = torch.arange(width * size, device="cuda"), s["lengths"][b]
        seen = place < length
        if s["window"]:
            seen = seen & (place >= length - s["window"])
        q = s["q"][b].float().reshape(H, group, dim)
        score = torch.where(seen, s["scale"] * (q @ keys.transpose(1, 2)), torch.full((), -math.inf, device="cuda"))
        top = score.amax(-1, keepdim=True)
        weight = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = weight.sum(-1, keepdim=True)
        mixed = weight @ torch.where(seen[:, None], values, torch.zeros((), device="cuda"))
        out[b] = (mixed / torch.where(total > 0, total, torch.ones_like(total))).reshape(s["heads"], dim)
    return out.to(s["q"].dtype)


def _act(v, name):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * 0.7071067811865476))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(0.7978845608028654 * (v + 0.044715 * v * v * v)))
    return v


def _plain_product(s):
    R, half = s["w_codes"].shape
    rt, kt = (R + 127) // 128, (half // 16 + 3) // 4
    scales = s["w_scales"].reshape(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)[:R]
    v = s["x"].float() @ _decoded(s["w_codes"], scales, "mxfp4", 2 * half).t()
    if s["bias"] is not None:
        v = v + s["bias"]
    if s["glu"]:
        v = v.reshape(v.shape[0], -1, 2, 32)
        v = (_act(v[..., 0, :], s["act"]) * v[..., 1, :]).reshape(v.shape[0], -1)[:, : s["N"]]
    else:
        v = _act(v, s["act"])
    if s["residual"] is not None:
        v = s["residual"].float() + v
    return v.to(DTYPES[s["out"]])


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"rotary": _plain_rotary, "store": _plain_store, "attention": _plain_attention, "product": _plain_product}[op](s)
    B = _binding()
    if op == "rotary":
        return B.kroquant_rotary(s["q"], s["k"], s["positions"], s["frequencies"], axes=_axes(s), layout=s["layout"], inverse=s["inverse"])
    if op == "store":
        B.kroquant_cache_write(s["cache"], s["k_new"], s["v_new"], s["table"], offsets=s["new_offsets"], starts=s["starts"])
        return B.kroquant_cache_read(s["cache"], s["table"], s["total"], offsets=s["all_offsets"], dtype=DTYPES[s["dtype"]])
    if op == "attention":
        return B.kroquant_cache_attention(s["q"], s["cache"], s["table"], s["lengths"], scale=s["scale"], window=s["window"])
    return B.kroquant_linear_w4a16(s["x"], s["w_codes"], s["w_scales"], features=s["N"], bias=s["bias"], activation=s["act"],
                                   glu=s["glu"], residual=s["residual"], out_dtype=DTYPES[s["out"]])


# -------------------------------------------------------------------------------------------------------------- 64 bits
def _format_values(form, device):
    """Non-negative values of the format in order, float64, from its definition; an index is even where the mantissa is."""
    bits, bias, codes = (3, 7, 127) if form == "mxfp8" else (1, 1, 8)
    out = []
    for c in range(codes):
        e, m = c >> bits, c & ((1 << bits) - 1)
        out.append(m * 2.0 ** (1 - bias - bits) if e == 0 else (1 + m / 2 ** bits) * 2.0 ** (e - bias))
    return torch.tensor(out, dtype=torch.float64, device=device)


def _exact_quantized(x, form):
    """x [..., dim] -> the values it becomes in the cache, float64."""
    if form == "16bit":
        return x.double()
    dim, values = x.shape[-1], _format_values(form, x.device)
    blocks = torch.nn.functional.pad(x.double(), (0, -dim % 32)).reshape(*x.shape[:-1], -1, 32)
    amax = blocks.abs().amax(-1, keepdim=True)
    top = math.floor(math.log2(float(values[-1])))
    power = torch.floor(torch.log2(torch.where(amax > 0, amax, torch.ones_like(amax)))) - top
    scale = torch.exp2(power.clamp(-127, 127))
    size = (blocks / scale).abs()
    upper = torch.searchsorted(values, size).clamp(1, len(values) - 1)
    below, above = values[upper - 1], values[upper]
    nearer_above = (size - below > above - size) | ((size - below == above - size) & (upper % 2 == 0))
    out = torch.where(nearer_above, above, below) * torch.sign(blocks) * scale
    return out.flatten(-2)[..., :dim]


def _exact_rows(codes, scales, form, dim):
    """What rows of the cache stand for, float64."""
    if form == "16bit":
        return codes[..., :dim].double()
    values, half = _format_values(form, codes.device), 128 if form == "mxfp8" else 8
    if form == "mxfp4":
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    code = codes[..., :dim].long()
    sign = torch.where(code >= half, -1.0, 1.0).double()
    power = scales.double().repeat_interleave(32, -1)[..., :dim] - 127
    return sign * values[code % half] * torch.exp2(power)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "rotary":
        first, second = _pair_channels(case, "cuda")
        column = [i for i, a in enumerate(_axes(case)) for _ in range(a // 2)]
        turn = torch.complex(torch.zeros((), dtype=torch.float64, device="cuda"), s["positions"][:, column].double() * s["frequencies"]).exp()
        if case["inverse"]:
            turn = turn.conj()
        out = []
        for x in (s["q"].double(), s["k"].double()):
            z = torch.complex(x[..., first], x[..., second]) * turn[:, None, :]
            x[..., first], x[..., second] = z.real, z.imag
            out.append(x)
        return tuple(out)
    if op == "store":
        size, dim, form, out = case["page_size"], case["dim"], case["format"], []
        for name in ("k", "v"):
            new, rows, at = _exact_quantized(s[name + "_new"], form), [], 0
            for b, (h, n) in enumerate(_chunks(case)):
                pages = s["table"][b, : (h + size - 1) // size].long()
                scales = None if form == "16bit" else s[name + "_scales"][pages].transpose(1, 2).flatten(0, 1)[:h]
                rows += [_exact_rows(s[name][pages].transpose(1, 2).flatten(0, 1)[:h], scales, form, dim), new[at : at + n]]
                at += n
            out.append(torch.cat(rows))
        return tuple(out)
    if op == "attention":
        size, dim, form, H = case["page_size"], case["dim"], case["format"], case["kv_heads"]
        out = torch.zeros(case["sequences"], case["heads"], dim, dtype=torch.float64, device="cuda")
        for b, n in enumerate(_lengths(case)):
            first = max(0, n - case["window"]) if case["window"] else 0
            if n == 0:
                continue
            p0 = first // size
            pages = s["table"][b, p0 : (n + size - 1) // size].long()
            kv = []
            for name in ("k", "v"):
                scales = None if form == "16bit" else s[name + "_scales"][pages].transpose(0, 1).flatten(1, 2)[:, first - p0 * size : n - p0 * size]
                kv.append(_exact_rows(s[name][pages].transpose(0, 1).flatten(1, 2)[:, first - p0 * size : n - p0 * size], scales, form, dim))
            q = s["q"][b].double().view(H, -1, dim)
            out[b] = (torch.softmax(s["scale"] * torch.bmm(q, kv[0].mT), -1).bmm(kv[1])).reshape(-1, dim)
        return out
    R, half = s["w_codes"].shape
    t, j = torch.arange(R, device="cuda")[:, None], torch.arange(half // 16, device="cuda")[None, :]
    at = ((t // 128) * ((half // 16 + 3) // 4) + j // 4) * 512 + (t % 32) * 16 + ((t % 128) // 32) * 4 + j % 4
    v = s["x"].double() @ _exact_rows(s["w_codes"], s["w_scales"][at], "mxfp4", 2 * half).T
    if s["bias"] is not None:
        v = v + s["bias"].double()
    name = case["act"]

    def f(z):
        if name == "relu":
            return z.clamp_min(0)
        if name == "silu":
            return z * torch.sigmoid(z)
        if name == "gelu":
            return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
        if name == "gelu_tanh":
            return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return z

    if case["glu"]:
        columns = torch.arange(case["N"], device="cuda")
        gate = columns // 32 * 64 + columns % 32
        v = f(v[:, gate]) * v[:, gate + 32]
    else:
        v = f(v)
    return v if s["residual"] is None else v + s["residual"].double()
