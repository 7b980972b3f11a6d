"""Rows in 4 bits from their definition, in 64 bits, and the bytes of their pages; the rotation.

Group of 32 channels x: range = max(x, 0) - min(x, 0) (rounded to 32 bits), s the least number of 4 significant bits,
2^-100 at least, with 15 s >= range, z = round(-min(x, 0) / s), n = clamp(round(x / s) + z, 0, 15), ties to even; the value is
s (n - z).  In 64 bits the quotients are right to the last of 53 bits, and a quotient that is not a tie is 2^-9 away from one."""
import torch


def quantise(x):
    """x [..., 128] bf16 -> codes int64 [..., 4, 32], s and z float64 [..., 4]; s is NaN for a group that is not finite."""
    g = x.double().unflatten(-1, (4, 32))
    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    low, high = torch.minimum(g.amin(-1), zero), torch.maximum(g.amax(-1), zero)
    wide = (high.float() - low.float()).double()
    fine = wide.isfinite() & g.isfinite().all(-1)
    w = torch.where(fine, wide, 1.0)
    low = torch.where(fine, low, 0.0)
    m = 8 * 2.0 ** -103 * torch.ones_like(w)  # 2^-100, as 8 units
    unit = torch.full_like(w, 2.0 ** -103)
    for _ in range(240):  # the unit doubles until 15 units can reach the range with 4 bits
        more = 15 * 15 * unit < w
        unit = torch.where(more, unit * 2, unit)
    for count in range(15, 7, -1):  # the least count of units that does
        m = torch.where(15 * count * unit >= w, count * unit, m)
    s = torch.where(w <= 15 * 2.0 ** -100, 2.0 ** -100, m)
    z = torch.round(-low / s)
    n = (torch.round(torch.where(fine[..., None], g, 0.0) / s[..., None]) + z[..., None]).clamp(0, 15)
    nan = torch.full_like(s, float("nan"))
    return torch.where(fine[..., None], n, 0).long(), torch.where(fine, s, nan), torch.where(fine, z, 0.0)


def values(codes, s, z):
    return ((codes - z[..., None]) * s[..., None]).flatten(-2)


def row_bytes(codes, s, z):
    """uint8 [..., 64] codes (4 groups of 16 bytes) and [..., 8] scales."""
    c = codes.unflatten(-1, (4, 8))
    word = torch.zeros(c.shape[:-1], dtype=torch.int64, device=c.device)
    for i in range(8):
        word |= c[..., i] << (4 * (i // 2 + 4 * (i % 2)))
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32).contiguous()
    scale = (s.to(torch.bfloat16).view(torch.int16) & 0x7FFF).to(torch.int16) | z.to(torch.int16)
    scale = torch.where(s.isnan(), torch.tensor(0x7FC0, dtype=torch.int16, device=s.device), scale).contiguous()
    return word.view(torch.uint8).flatten(-2), scale.view(torch.uint8)


def put(pages, page_size, slots, rows, which):
    """Rows [T, H, 128] (bf16) into the K (0) or V (1) blocks of pages [num_pages, H, 2, page_size * 72]; -1 is skipped."""
    codes, scales = row_bytes(*quantise(rows))
    t = (slots >= 0).nonzero()[:, 0]
    page, row = slots[t].long() // page_size, slots[t].long() % page_size
    P = page_size
    block = pages[:, :, which]
    block[..., :64 * P].unflatten(-1, (4, P, 16))[page, :, :, row] = codes[t].unflatten(-1, (4, 16))
    block[..., 64 * P:].unflatten(-1, (P, 8))[page, :, row] = scales[t]


def held(x):
    """The values (bf16 numbers, in bf16) that 4 bits hold of x."""
    return values(*quantise(x)).to(torch.bfloat16)


def rotate(x, cos_sin, positions, interleaved=False):
    """x [T, H, 128] bf16 -> bf16: exact in 64 bits, rounded to 32 and then to bf16."""
    rd = cos_sin.shape[1]
    cos, sin = (a[:, None] for a in cos_sin.double()[positions.long()].split(rd // 2, 1))
    y = x.double().clone()
    lead = torch.arange(rd // 2, device=x.device)
    ia, ib = (2 * lead, 2 * lead + 1) if interleaved else (lead, lead + rd // 2)
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = a * cos - b * sin, b * cos + a * sin
    return y.float().to(torch.bfloat16)
