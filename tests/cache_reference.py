"""The paged cache in plain terms, float64, for the tests: the formats from their definitions, one row at a time."""
import torch


def grid(form):
    """Non-negative values of E4M3 or E2M1 in order; the index is even where the mantissa is."""
    if form == "mxfp8":
        return torch.tensor([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64)
    return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def quantized(x, form):
    """x [..., d] (CPU) -> (values it becomes, codes [..., C], scale bytes [..., C / 32]), C = d filled up to a multiple of 32."""
    d = x.shape[-1]
    blocks = torch.nn.functional.pad(x.double(), (0, -d % 32)).unflatten(-1, (-1, 32))
    amax = blocks.abs().amax(-1)
    exponent = torch.frexp(amax)[1] - 1
    byte = torch.where(amax > 0, (exponent - (8 if form == "mxfp8" else 2) + 127).clamp(0, 254), torch.zeros_like(exponent))
    scale = torch.exp2(byte.double() - 127)[..., None]
    v, size = grid(form), (blocks / scale).abs()
    up = torch.searchsorted(v, size).clamp(1, len(v) - 1)
    low, high = v[up - 1], v[up]
    to_high = (size - low > high - size) | ((size - low == high - size) & (up % 2 == 0))
    index = torch.where(to_high, up, up - 1)
    negative = torch.signbit(blocks)
    values = v[index] * torch.where(negative, -1.0, 1.0) * scale
    codes = index + negative * (128 if form == "mxfp8" else 8)
    return values.flatten(-2)[..., :d], codes.flatten(-2), byte


def decoded(codes, scales, form, d):
    """Rows of a cache's buffers (any device) -> float64 values [..., d]."""
    if form == "16bit":
        return codes[..., :d].double()
    v, half = grid(form).to(codes.device), 128 if form == "mxfp8" else 8
    if form == "mxfp8":
        v = torch.cat([v, torch.full((1,), float("nan"), dtype=torch.float64, device=codes.device)])
    else:
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    code = codes.long()
    out = v[code % half] * torch.where(code >= half, -1.0, 1.0).double()
    power = torch.exp2(scales.double() - 127).repeat_interleave(32, -1)[..., : out.shape[-1]]
    return (out * power)[..., :d]


def gather(cache, table_row, first, end):
    """Keys and values of positions first .. end - 1 of one sequence, float64 [heads, n, d], and which of them have a place."""
    t = torch.arange(first, end, device=cache.device)
    entry = t // cache.page_size
    page = table_row.to(cache.device)[entry.clamp_max(table_row.numel() - 1)].long() if table_row.numel() else torch.full_like(t, -1)
    live = (entry < table_row.numel()) & (page >= 0) & (page < cache.pages)
    page, slot = torch.where(live, page, torch.zeros_like(page)), t % cache.page_size
    out = []
    for name in ("k", "v"):
        rows = getattr(cache, name)[page, :, slot]                       # [n, heads, row]
        scales = getattr(cache, name + "_scales")
        rows = decoded(rows, None if scales is None else scales[page, :, slot], cache.format, cache.head_dim)
        out.append(torch.where(live[:, None, None], rows, torch.zeros_like(rows)).transpose(0, 1))
    return out[0], out[1], live
