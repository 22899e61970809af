"""Operators of a quantized transformer block around the MXFP4 product: cases, inputs, plain forms, 64-bit values.

Three operators that stand between one low-bit product and the next:

* ``linear``   out = r * residual + gate * act(A W^T + bias), A and W in MXFP4 (packed E2M1 codes, one E8M0 byte per
               32 channels in the 128 x 4 tiled layout), optionally with the gated activation act(g) * u;
* ``grouped``  the same product with one weight per expert, the rows of A sorted by expert, ragged group sizes;
* ``norm``     h = r * x + gate * post_norm(y);  n = norm(h) * weight * (1 + scale) + shift;
  ``norm_grad`` its backward pass.

The plain form (``own`` false) is elementary torch arithmetic in 32 bits with one rounding at the end; ``exact`` computes
the same definitions in 64 bits and is written separately.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6

_package = None


def _binding():
    global _package
    if _package is None:
        from paper_2607_21446_b200 import binding
        _package = binding
    return _package


# ---------------------------------------------------------------------------------------------------------------- cases
def _linear(name, M, N, K, act="none", glu=False, bias=True, gates=0, residual=False, out="bf16"):
    return {"name": name, "op": "linear", "M": M, "N": N, "K": K, "act": act, "glu": glu, "bias": bias, "gates": gates,
            "residual": residual, "out": out}


def _grouped(name, T, E, N, K, act="none", glu=False, bias=False, weighted=False, spread="even", out="bf16"):
    return {"name": name, "op": "grouped", "T": T, "E": E, "N": N, "K": K, "act": act, "glu": glu, "bias": bias,
            "weighted": weighted, "spread": spread, "out": out}


def _norm(name, op, rows, d, batches=1, norm="rms", post="none", modulated=False, gated=False, stream="bf16", branch="bf16"):
    return {"name": name, "op": op, "rows": rows, "d": d, "batches": batches, "norm": norm, "post": post,
            "modulated": modulated, "gated": gated, "stream": stream, "branch": branch}


def listed():
    return [
        # the modulation layer of a 1152-wide block (one conditioning row -> six vectors of 1152), float out: latency
        _linear("modulation_1_row", 1, 6912, 1152, out="f32"),
        # a decode step of 24 sequences through a projection back into the residual stream
        _linear("decode_24_rows", 24, 4096, 4096, residual=True),
        # the first feed-forward product of a 2240-wide block on a ragged number of tokens, odd feature count
        _linear("ffn_in_ragged", 4099, 5601, 2240, act="gelu_tanh", out="f16"),
        # the largest: a 4608-wide feed-forward entry, gated residual per sample of a batch of four
        _linear("ffn_large_gated", 16384, 12288, 4608, act="none", gates=4, residual=True),
        # experts in decode: eight tokens with two experts each, gated activation; the weights are what is read
        _grouped("experts_decode", 16, 8, 5632, 4096, act="silu", glu=True, spread="ragged"),
        # many small groups (some of them empty) on the way back, weighted by the router
        _grouped("experts_small_groups", 1030, 32, 2240, 5600, weighted=True, spread="ragged"),
        # experts over a long batch, gated activation
        _grouped("experts_long", 16384, 8, 5632, 4096, act="silu", glu=True, spread="even"),
        # one token through the norm between two sub-blocks
        _norm("norm_one_token", "norm", 1, 4096),
        # the adaptive layer norm of a 2240-wide block behind its gated attention branch, two samples
        _norm("norm_adaptive", "norm", 8192, 2240, batches=2, norm="layer", modulated=True, gated=True),
        # norms before and after the block, 32-bit residual stream, wide rows
        _norm("norm_sandwich_wide", "norm", 16385, 5600, norm="rms", post="rms", stream="f32"),
        # backward: a short ragged batch with an odd width
        _norm("norm_grad_odd", "norm_grad", 517, 1153, norm="rms", post="rms", stream="f16", branch="f16"),
        # backward of the adaptive layer norm over a long batch of four samples
        _norm("norm_grad_long", "norm_grad", 16384, 4608, batches=4, norm="layer", modulated=True, gated=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["linear", "grouped", "norm", "norm_grad"])
    act, glu = rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.4
    if op == "linear":
        while True:
            M, N, K = _log(rng, 1, 16384), _log(rng, 32, 12288), 32 * _log(rng, 4, 384)
            if M * N * (2 if glu else 1) * K <= 16384 * 12288 * 4608:
                break
        gates = rng.choice([0, 0, 1, 2])
        if gates == 2 and M % 2:
            gates = 1
        c = _linear("", M, N, K, act, glu, rng.random() < 0.5, gates, rng.random() < 0.5, rng.choice(["bf16", "f16", "f32"]))
    elif op == "grouped":
        while True:
            T, E, N, K = _log(rng, 1, 16384), _log(rng, 1, 64), _log(rng, 64, 8192), 32 * _log(rng, 8, 256)
            spread, rows = rng.choice(["even", "ragged", "one"]), N * (2 if glu else 1)
            if E * rows * K <= 4e8 and E * max(_group_sizes(T, E, spread)) * rows * K <= 8e11:
                break
        c = _grouped("", T, E, N, K, act, glu, rng.random() < 0.5, rng.random() < 0.5, spread, rng.choice(["bf16", "f16", "f32"]))
    else:
        while True:
            rows, d = _log(rng, 1, 16384), _log(rng, 64, 12288)
            if rows * d <= 16384 * 4608:
                break
        if rng.random() < 0.75:
            d = max(32, d // 32 * 32)
        batches = rng.choice([b for b in (1, 2, 3, 8) if rows % b == 0])
        branch = rng.choice(["bf16", "f16"])
        c = _norm("", op, rows, d, batches, rng.choice(["rms", "layer"]), rng.choice(["none", "rms", "layer"]),
                  rng.random() < 0.6, rng.random() < 0.6, rng.choice([branch, branch, "f32"]), branch)
    del c["name"]
    return c


def _group_sizes(T, E, spread):
    """Rows per expert; which expert gets which size is drawn from the seed."""
    if spread == "one":
        return [T] + [0] * (E - 1)
    if spread == "even":
        share = [1.0 + 0.15 * ((7 * i) % 5 - 2) for i in range(E)]
    else:                                              # a few large groups, many small ones, every fourth empty
        share = [0.0 if E >= 4 and i % 4 == 3 else 1.0 / math.sqrt(i + 1.0) for i in range(E)]
    total, sizes = sum(share), []
    for s in share:
        sizes.append(int(T * s / total))
    for k in range(T - sum(sizes)):
        live = [i for i in range(E) if share[i] > 0]
        sizes[live[k % len(live)]] += 1
    return sizes


def _weight_rows(case):
    """Rows of the stored weight: a gated activation interleaves 32 gate rows with 32 value rows."""
    return 64 * ((case["N"] + 31) // 32) if case["glu"] else case["N"]


def work(case):
    op = case["op"]
    if op == "linear":
        M, N, K, R = case["M"], case["N"], case["K"], _weight_rows(case)
        size = SIZES[case["out"]]
        nbytes = (M + R) * K * (0.5 + 1 / 32) + M * N * size * (2 if case["residual"] else 1)
        nbytes += 4 * R * case["bias"] + 4 * N * case["gates"]
        return {"bytes": nbytes, "flops": 2.0 * M * R * K}
    if op == "grouped":
        T, N, K, R = case["T"], case["N"], case["K"], _weight_rows(case)
        live = sum(1 for s in _group_sizes(T, case["E"], case["spread"]) if s)
        nbytes = (T + live * R) * K * (0.5 + 1 / 32) + T * N * SIZES[case["out"]] + 4 * live * R * case["bias"] + 4 * T * case["weighted"]
        return {"bytes": nbytes, "flops": 2.0 * T * R * K}
    n = case["rows"] * case["d"]
    s, b = SIZES[case["stream"]], SIZES[case["branch"]]
    if op == "norm":
        return {"bytes": n * (2 * s + 2 * b), "flops": 12.0 * n}
    return {"bytes": n * (3 * s + 3 * b), "flops": 30.0 * n}


# --------------------------------------------------------------------------------------------------------------- inputs
def _encode(x):
    """float [..., R, K] -> packed E2M1 codes uint8 [..., R, K/2] and E8M0 bytes uint8 [..., R, K/32]."""
    blocks = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    amax = blocks.abs().amax(-1)
    exponent = torch.where(amax > 0, torch.floor(torch.log2(amax.clamp_min(1e-30))) - 2, torch.full_like(amax, -127.0))
    scaled = blocks * torch.exp2(-exponent)[..., None]
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    code = torch.bucketize(scaled.abs(), edges).to(torch.uint8) | ((scaled < 0).to(torch.uint8) << 3)
    code = code.reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (exponent + 127).to(torch.uint8)


def _tile(scales):
    """E8M0 bytes [R, K/32] -> the 128 x 4 tiled layout, flat."""
    R, B = scales.shape
    rt, kt = (R + 127) // 128, (B + 3) // 4
    full = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=scales.device)
    full[:R, :B] = scales
    return full.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _activations(rows, K, g):
    x = torch.randn(rows, K, device="cuda", generator=g)
    loud = torch.randint(0, K, (max(1, K // 100),), device="cuda", generator=g)
    x[:, loud] *= 20.0
    return x


def _weights(rows, K, g):
    return torch.randn(rows, K, device="cuda", generator=g) / math.sqrt(K)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op = case["op"]
    state = dict(case)
    if op in ("linear", "grouped"):
        N, K, R = case["N"], case["K"], _weight_rows(case)
        rows = case["M"] if op == "linear" else case["T"]
        dtype = DTYPES[case["out"]]
        codes, scales = _encode(_activations(rows, K, g))
        state["a_codes"], state["a_scales"] = codes, _tile(scales)
        count = 1 if op == "linear" else case["E"]
        w_codes = torch.empty(count, R, K // 2, dtype=torch.uint8, device="cuda")
        w_scales = []
        for e in range(count):
            w_codes[e], s = _encode(_weights(R, K, g))
            w_scales.append(_tile(s))
        state["w_codes"], state["w_scales"] = w_codes, torch.stack(w_scales)
        state["bias"] = 0.2 * torch.randn(count, R, device="cuda", generator=g) if case["bias"] else None
        if op == "linear":
            state["w_codes"], state["w_scales"] = w_codes[0], state["w_scales"][0]
            state["bias"] = state["bias"][0] if case["bias"] else None
            state["gate"] = torch.randn(case["gates"], N, device="cuda", generator=g) if case["gates"] else None
            state["residual"] = torch.randn(rows, N, device="cuda", generator=g).to(dtype) if case["residual"] else None
        else:
            sizes = torch.tensor(_group_sizes(rows, count, case["spread"]))
            sizes = sizes[torch.randperm(count, generator=torch.Generator().manual_seed(int(seed)))]
            state["capacity"] = int(sizes.max())
            state["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), sizes.cumsum(0)]).to(torch.int32).cuda()
            state["row_scale"] = torch.rand(rows, device="cuda", generator=g) if case["weighted"] else None
        return state
    rows, d, batches = case["rows"], case["d"], case["batches"]
    stream, branch = DTYPES[case["stream"]], DTYPES[case["branch"]]

    def normal(dtype, *shape, gain=1.0, mean=0.0):
        return (gain * torch.randn(*shape, device="cuda", generator=g) + mean).to(dtype)

    loud = torch.ones(d, device="cuda")
    loud[torch.randint(0, d, (max(1, d // 100),), device="cuda", generator=g)] = 8.0
    state["y"] = normal(branch, rows, d, mean=0.1)
    state["weight"] = None if case["modulated"] else normal(torch.float32, d, gain=0.2, mean=1.0)
    state["scale"] = normal(torch.float32, batches, d, gain=0.3) if case["modulated"] else None
    state["shift"] = normal(torch.float32, batches, d, gain=0.3) if case["modulated"] else None
    state["gate"] = normal(torch.float32, batches, d, gain=0.5) if case["gated"] else None
    state["post_weight"] = normal(torch.float32, d, gain=0.2, mean=1.0) if case["post"] != "none" else None
    state["residual_scale"] = 1.0
    x = (torch.randn(rows, d, device="cuda", generator=g) + 0.2) * loud
    if op == "norm":
        state["x"] = x.to(stream)
    else:
        state["h"] = x.to(stream)
        state["dn"] = normal(branch, rows, d, gain=0.1)
        state["dh"] = normal(stream, rows, d, gain=0.1)
    return state


# ----------------------------------------------------------------------------------------------------------- plain form
def _decode(codes, scales):
    """codes [R, K/2] and tiled scales -> float32 [R, K]."""
    R, half = codes.shape
    rt, kt = (R + 127) // 128, (half // 16 + 3) // 4
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    grid = torch.cat([grid, -grid])
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)            # byte -> (low code, high code)
    values = pairs[codes.int()].reshape(R, half // 16, 32)
    rows = scales.reshape(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)[:R, : half // 16]
    return (values * torch.exp2(rows.float() - 127)[..., None]).reshape(R, 2 * half)


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


def _activated(v, act, glu, N):
    """v [..., R] of the stored weight's rows -> [..., N]."""
    if not glu:
        return _act(v, act)
    v = v.reshape(*v.shape[:-1], -1, 2, 32)
    return (_act(v[..., 0, :], act) * v[..., 1, :]).reshape(*v.shape[:-3], -1)[..., :N]


def _plain_linear(s):
    v = _decode(s["a_codes"], s["a_scales"]) @ _decode(s["w_codes"], s["w_scales"]).t()
    if s["bias"] is not None:
        v = v + s["bias"]
    v = _activated(v, s["act"], s["glu"], s["N"])
    if s["gate"] is not None:
        v = (v.reshape(s["gates"], -1, s["N"]) * s["gate"][:, None, :]).reshape(-1, s["N"])
    if s["residual"] is not None:
        v = s["residual"].float() + v
    return v.to(DTYPES[s["out"]])


def _plain_grouped(s):
    T, E, cap, K = s["T"], s["E"], s["capacity"], s["K"]
    R = s["w_codes"].shape[1]
    a = _decode(s["a_codes"], s["a_scales"])
    kt = (K // 32 + 3) // 4
    tiles = s["w_scales"].reshape(E * ((R + 127) // 128), kt, 32, 4, 4).permute(0, 3, 2, 1, 4)
    tiles = tiles.reshape(E, -1, kt * 4)[:, :R, : K // 32]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=a.device)
    grid = torch.cat([grid, -grid])
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)
    w = (pairs[s["w_codes"].int()].reshape(E, R, K // 32, 32) * torch.exp2(tiles.float() - 127)[..., None]).reshape(E, R, K)
    start, row = s["offsets"][:-1].long(), torch.arange(T, device=a.device)
    expert = (row[:, None] >= s["offsets"][None, 1:]).sum(1)
    place = expert * cap + (row - start[expert])
    padded = torch.zeros(E * cap, K, device=a.device)
    padded[place] = a
    v = torch.bmm(padded.view(E, cap, K), w.transpose(1, 2)).reshape(E * cap, R)[place]
    if s["bias"] is not None:
        v = v + s["bias"][expert]
    v = _activated(v, s["act"], s["glu"], s["N"])
    if s["row_scale"] is not None:
        v = v * s["row_scale"][:, None]
    return v.to(DTYPES[s["out"]])


def _statistics(v, kind):
    """float rows -> (normalised rows, 1 / deviation)."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    inverse = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * inverse, inverse


def _by_batch(vector, rows, batches):
    return vector[:, None, :].expand(batches, rows // batches, vector.shape[-1]).reshape(rows, -1)


def _plain_norm(s):
    rows, batches = s["rows"], s["batches"]
    y = s["y"].float()
    if s["post"] != "none":
        y = _statistics(y, s["post"])[0] * s["post_weight"]
    if s["gate"] is not None:
        y = y * _by_batch(s["gate"], rows, batches)
    h = s["residual_scale"] * s["x"].float() + y
    n = _statistics(h, s["norm"])[0]
    if s["weight"] is not None:
        n = n * s["weight"]
    if s["scale"] is not None:
        n = n * (1 + _by_batch(s["scale"], rows, batches)) + _by_batch(s["shift"], rows, batches)
    return h.to(s["x"].dtype), n.to(s["y"].dtype)


def _norm_backward(g, xhat, inverse, kind):
    g = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if kind == "layer":
        g = g - g.mean(-1, keepdim=True)
    return g * inverse


def _plain_norm_grad(s):
    rows, batches, d = s["rows"], s["batches"], s["d"]
    dn, h, y = s["dn"].float(), s["h"].float(), s["y"].float()
    xhat, inverse = _statistics(h, s["norm"])
    out, g = {}, dn
    if s["weight"] is not None:
        out["dweight"] = (dn * xhat).sum(0)
        g = dn * s["weight"]
    if s["scale"] is not None:
        out["dscale"] = (dn * xhat).reshape(batches, -1, d).sum(1)
        out["dshift"] = dn.reshape(batches, -1, d).sum(1)
        g = dn * (1 + _by_batch(s["scale"], rows, batches))
    dh = s["dh"].float() + _norm_backward(g, xhat, inverse, s["norm"])
    out["dx"] = (s["residual_scale"] * dh).to(s["h"].dtype)
    dr, r = dh, y
    if s["post"] != "none":
        yhat, yinverse = _statistics(y, s["post"])
        r = yhat * s["post_weight"]
    if s["gate"] is not None:
        out["dgate"] = (dh * r).reshape(batches, -1, d).sum(1)
        dr = dh * _by_batch(s["gate"], rows, batches)
    if s["post"] != "none":
        out["dpost_weight"] = (dr * yhat).sum(0)
        dr = _norm_backward(dr * s["post_weight"], yhat, yinverse, s["post"])
    out["dy"] = dr.to(s["y"].dtype)
    return out


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"linear": _plain_linear, "grouped": _plain_grouped, "norm": _plain_norm, "norm_grad": _plain_norm_grad}[op](s)
    B = _binding()
    if op == "linear":
        return B.kroquant_linear_mxfp4(s["a_codes"], s["a_scales"], s["w_codes"], s["w_scales"], features=s["N"], bias=s["bias"],
                                       activation=s["act"], glu=s["glu"], gate=s["gate"], residual=s["residual"],
                                       out_dtype=DTYPES[s["out"]])
    if op == "grouped":
        return B.kroquant_linear_mxfp4_grouped(s["a_codes"], s["a_scales"], s["w_codes"], s["w_scales"], s["offsets"],
                                               features=s["N"], bias=s["bias"], activation=s["act"], glu=s["glu"],
                                               row_scale=s["row_scale"], out_dtype=DTYPES[s["out"]])
    given = {k: s[k] for k in ("gate", "post_weight", "weight", "scale", "shift", "residual_scale")}
    if op == "norm":
        return B.kroquant_norm_residual(s["x"], s["y"], norm=s["norm"], post_norm=s["post"], eps=EPS, **given)
    return B.kroquant_norm_residual_grad(s["dn"], s["h"], dh=s["dh"], y=s["y"], norm=s["norm"], post_norm=s["post"], eps=EPS, **given)


# -------------------------------------------------------------------------------------------------------------- 64 bits
def _exact_values(codes, scales):
    """The values that codes and tiled scale bytes stand for, from the formats' definitions, float64."""
    R, half = codes.shape
    code = torch.empty(R, 2 * half, dtype=torch.uint8, device=codes.device)
    code[:, 0::2], code[:, 1::2] = codes & 15, codes >> 4
    exponent, mantissa = ((code >> 1) & 3).double(), (code & 1).double()
    size = torch.where(exponent == 0, 0.5 * mantissa, torch.exp2(exponent - 1) * (1 + 0.5 * mantissa))
    size = torch.where(code >= 8, -size, size)
    t = torch.arange(R, device=codes.device)[:, None]
    j = torch.arange(half // 16, device=codes.device)[None, :]
    at = ((t // 128) * ((half // 16 + 3) // 4) + j // 4) * 512 + (t % 32) * 16 + ((t % 128) // 32) * 4 + j % 4
    byte = scales.reshape(-1)[at.reshape(-1)].reshape(R, half // 16).double()
    return size * torch.exp2(byte - 127).repeat_interleave(32, 1)


def _exact_activation(v, case):
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

    if not case["glu"]:
        return f(v)
    columns = torch.arange(case["N"], device=v.device)
    first = columns // 32 * 64 + columns % 32
    return f(v[:, first]) * v[:, first + 32]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "linear":
        v = _exact_values(s["a_codes"], s["a_scales"]) @ _exact_values(s["w_codes"], s["w_scales"]).t()
        v = _exact_activation(v if s["bias"] is None else v + s["bias"].double(), case)
        if s["gate"] is not None:
            v = v * s["gate"].double().repeat_interleave(case["M"] // case["gates"], 0)
        return v if s["residual"] is None else v + s["residual"].double()
    if op == "grouped":
        a, bounds = _exact_values(s["a_codes"], s["a_scales"]), s["offsets"].tolist()
        out = torch.zeros(case["T"], case["N"], dtype=torch.float64, device="cuda")
        for e in range(case["E"]):
            lo, hi = bounds[e], bounds[e + 1]
            if hi > lo:
                v = a[lo:hi] @ _exact_values(s["w_codes"][e], s["w_scales"][e]).t()
                out[lo:hi] = _exact_activation(v if s["bias"] is None else v + s["bias"][e].double(), case)
        return out if s["row_scale"] is None else out * s["row_scale"].double()[:, None]
    if case["rows"] * case["d"] > 2e8:
        return None
    d, per = case["d"], case["rows"] // case["batches"]
    wide = {k: (v.double() if isinstance(v, torch.Tensor) else v) for k, v in s.items()}

    def vector(name, default):
        v = wide[name]
        if v is None:
            return torch.full((1, d), default, dtype=torch.float64, device="cuda")
        return v[None, :] if v.dim() == 1 else v.repeat_interleave(per, 0)

    def normal(v, kind):
        centre = v.mean(1, keepdim=True) if kind == "layer" else 0.0
        deviation = ((v - centre).square().sum(1, keepdim=True) / d + EPS).sqrt()
        return (v - centre) / deviation, deviation

    gate, post, y = vector("gate", 1.0), vector("post_weight", 1.0), wide["y"]
    multiplier, shift = vector("weight", 1.0) * (1 + vector("scale", 0.0)), vector("shift", 0.0)
    yhat, ydev = normal(y, case["post"]) if case["post"] != "none" else (y, None)
    if op == "norm":
        h = wide["residual_scale"] * wide["x"] + gate * yhat * post
        return h, normal(h, case["norm"])[0] * multiplier + shift
    hhat, hdev = normal(wide["h"], case["norm"])

    def back(cotangent, hat, dev, kind):
        along = (cotangent * hat).sum(1, keepdim=True) / d
        level = cotangent.sum(1, keepdim=True) / d if kind == "layer" else 0.0
        return (cotangent - level - hat * along) / dev

    dn, grads = wide["dn"], {}
    total = wide["dh"] + back(dn * multiplier, hhat, hdev, case["norm"])
    if wide["weight"] is not None:
        grads["dweight"] = torch.einsum("td,td->d", dn, hhat)
    if wide["scale"] is not None:
        grads["dscale"] = torch.einsum("btd,btd->bd", dn.view(-1, per, d), hhat.view(-1, per, d))
        grads["dshift"] = dn.view(-1, per, d).sum(1)
    grads["dx"] = wide["residual_scale"] * total
    if wide["gate"] is not None:
        grads["dgate"] = torch.einsum("btd,btd->bd", total.view(-1, per, d), (yhat * post).view(-1, per, d))
    if case["post"] != "none":
        grads["dpost_weight"] = (total * gate * yhat).sum(0)
        grads["dy"] = back(total * gate * post, yhat, ydev, case["post"])
    else:
        grads["dy"] = total * gate
    return grads
