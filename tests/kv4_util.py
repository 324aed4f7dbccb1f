"""The four-bit cache format in plain fp64, element by element, for the tests."""
import torch

LEVELS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def quantised(x):
    """What the format holds for rows x [..., d] (CPU), in fp64: NaN for blocks with a NaN or an
    infinity."""
    b = x.double().unflatten(-1, (-1, 32))
    finite = torch.isfinite(b).all(-1, keepdim=True)
    a = torch.where(finite, b, 0.0).abs()
    top = a.amax(-1, keepdim=True)
    byte = torch.full_like(top, 2.0)
    for e in range(2, 253):      # the smallest byte that does
        byte = torch.where((top <= 7 * 2.0 ** (e - 127)) & (byte == 2) & (top > 7 * 2.0 ** (e - 128)), float(e), byte)
    byte = torch.where(top > 7 * 2.0 ** (252 - 127), 252.0, byte)
    scale = torch.exp2(byte - 127)
    y = a / scale
    dist = (y[..., None] - LEVELS).abs()
    near = dist.amin(-1, keepdim=True)
    tie = dist == near
    index = torch.arange(8)
    # of two levels equally near, the one with the even code
    choice = torch.where(tie, torch.where(index % 2 == 0, 0, 1), 2).argmin(-1)
    v = torch.where(b < 0, -1.0, 1.0) * LEVELS[choice] * scale
    return torch.where(finite, v, float("nan")).flatten(-2)


def stored(cache, page, d, table, b, n):
    """fp64 keys and values [heads, n, d] of the first n tokens of sequence b (all on CPU), each
    element by its place in the page."""
    j = torch.arange(n)
    ids = table[b].long()[j // page] if table is not None else torch.full((n,), b)
    r, e = (j % page)[:, None], torch.arange(d)[None]
    a, t, g, i = r // 64, r % 64 // 16, r % 16 // 4, r % 4
    kc = r * (d // 2) + e // 2
    ks = page * d // 2 + ((a * (d // 32) + e // 32) * 16 + r % 16) * 4 + t
    vc = page * (d // 2 + d // 32) + ((r // 4 * (d // 4) + e // 4) * 4 + i) * 2 + e % 4 // 2
    vs = page * (d + d // 32) + (((a * (d // 32) + e // 32) * 4 + g) * 4 + t) * 4 + i
    out = []
    for code, scale in ((kc, ks), (vc, vs)):
        rows = cache[ids]                                  # [n, heads, bytes]
        c = rows.gather(2, code[:, None].expand(-1, rows.shape[1], -1)).long()
        s = rows.gather(2, scale[:, None].expand(-1, rows.shape[1], -1)).double()
        c = torch.where(e % 2 == 1, c >> 4, c & 15)
        v = torch.where(c >= 8, -1.0, 1.0) * LEVELS[c % 8] * torch.exp2(s - 127)
        out.append(torch.where(s == 255, float("nan"), v).transpose(0, 1))
    return out
