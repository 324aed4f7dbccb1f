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


U = 2.0 ** -24


def attention(q, K, V, seen, scale):
    """One head in fp64: q [n, d] over K, V [m, d] (CPU), row i sees the first seen[i] keys.
    (O, LSE, sum P |V|, the largest scale * sum |q k| of a row)."""
    hide = torch.arange(K.shape[0])[None] >= seen[:, None]
    s = (q @ K.t() * scale).masked_fill(hide, -torch.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(hide, 0.0, torch.exp(s - lse[:, None]))
    held = torch.isnan(V)
    V = torch.where(held, 0.0, V)
    o, mag = p @ V, p @ V.abs()
    o[(~hide).double() @ held.double() > 0] = torch.nan
    sizes = (q.abs() @ torch.nan_to_num(K).abs().t()).masked_fill(hide, 0)
    reach = sizes.amax(-1) * abs(scale) if K.shape[0] else sizes.sum(-1)
    empty = seen <= 0
    o[empty], mag[empty], lse[empty] = 0.0, 0.0, -torch.inf
    return o, lse, mag, reach


def attention_error(o, lse, ref, keys, d, half=U):
    """The largest shares that O and LSE (fp64) take of their bounds, or a text that says what is
    NaN or infinite where `ref` is not.

    A weight goes into the product with V as two bf16 numbers, of which the second leaves half a
    step of 2^-8 of a rest of at most 2^-9: 2^-18 of sum P |V|.  Scores are off by (d + 4) units of
    2^-24 of scale * sum |q k|, which weights and sums have; fp32 sums of n terms add n / 64 + 64
    units; the output's type adds half a step, `half` (fp32's)."""
    want, wl, mag, reach = ref
    for name, got, right in (("O", o, want), ("LSE", lse, wl)):
        for what, test in (("NaN", torch.isnan), ("infinite", torch.isinf)):
            if not torch.equal(test(got), test(right)):
                return f"{name}: {what} at {int((test(got) != test(right)).sum())} places"
    ds, sums = (d + 4) * U * reach, (keys / 64 + 64) * U
    live = torch.isfinite(wl)
    lim = (2.0 ** -18 + 2 * ds[:, None] + sums) * mag + half * want.abs() + 1e-30
    err = torch.nan_to_num((o - want).abs() / lim).amax().item() if o.numel() else 0.0
    lerr = ((lse - wl).abs() / (ds + sums + 4 * U * wl.abs()))[live]
    return err, lerr.amax().item() if lerr.numel() else 0.0
