"""The four-bit key/value cache on the GPU: what is written and read back equals the format's
definition exactly; the attention is checked against fp64 over the stored values.

Tolerance of the attention, per element: the weights are rounded to bf16 before they multiply V
(half a step, 2^-8 of sum P |V|); scores are off by at most (d + 4) units of 2^-24 relative to
scale * sum |q k|, which the weights inherit, and fp32 sums of up to n terms add n / 64 + 64 units;
a bf16 output adds half a step, 2^-8 |O|.  LSE has the same without the weights' rounding.
"""
import math

import pytest

from kv4_util import quantised, stored

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _say(*a):
    print(*a, flush=True)


def _pool(B, cap, page, Hk, d, gen, paged=True, spare=3, fill=0xFF):
    """A cache filled with `fill` bytes (255: what reads as NaN) and a shuffled page table."""
    import torch
    import paper_2606_07713_amd as moa
    each = -(-cap // page)
    n = B * each + spare if paged else B
    cache = moa.kv4_cache(n, Hk, page, d)
    cache.fill_(fill)
    table = torch.randperm(n, generator=gen)[:B * each].view(B, each).int().to("cuda") if paged else None
    return cache, table


def _ints(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# B, Hk, N, d, page, dtype, lens, new_lens
WRITES = [
    (1, 1, 1, 64, 64, "bf16", [1], None),
    (3, 2, 1, 128, 64, "bf16", [1, 64, 131], None),
    (2, 3, 130, 128, 128, "bf16", [130, 177], None),
    (2, 5, 67, 64, 192, "f32", [70, 500], [67, 13]),
    (3, 1, 9, 128, 64, "f32", [0, 5, 300], [0, 5, 9]),
    (2, 2, 5, 64, 64, "bf16", [3, 200], None),          # more rows than tokens: the first are before 0
]


@pytest.mark.parametrize("case", WRITES, ids=lambda c: "x".join(map(str, c[:5])) + "_" + c[5])
def test_write_and_read_back(case):
    import torch
    import paper_2606_07713_amd as moa
    B, Hk, N, d, page, dtype, lens, new = case
    _say(f"kv4 write {case}")
    gen = torch.Generator().manual_seed(5)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    cap = max(lens) + 1
    cache, table = _pool(B, cap, page, Hk, d, gen, fill=0x77)
    before = cache.cpu().clone()
    # blocks of very different size, ties, zeros
    x = [torch.randn((B, N, Hk, d), generator=gen) * torch.exp2(torch.randint(-20, 20, (B, N, Hk, 1), generator=gen).float())
         for _ in range(2)]
    x[0][..., :32] = torch.randint(-12, 13, (B, N, Hk, 32), generator=gen) / 4.0
    x[1][..., 32:] = 0
    k, v = (t.to(dt).to("cuda").transpose(1, 2) for t in x)
    moa.kv4_write(k, v, cache, _ints(lens), page_table=table, new_lens=None if new is None else _ints(new))
    odt = torch.float32 if dtype == "bf16" else torch.bfloat16
    ko = torch.full((B, Hk, N, d), 3.0, dtype=odt, device="cuda")
    vo = torch.full((B, N, Hk, d), 3.0, dtype=odt, device="cuda").transpose(1, 2)
    moa.kv4_read(cache, N, d, _ints(lens), page_table=table, new_lens=None if new is None else _ints(new), k_out=ko, v_out=vo)
    torch.cuda.synchronize()
    host, tab = cache.cpu(), table.cpu()
    touched = torch.zeros_like(before, dtype=torch.bool)
    for b in range(B):
        n = N if new is None else new[b]
        want = [quantised(t.cpu()[b]) for t in (k, v)]
        held = stored(host, page, d, tab, b, lens[b])
        for i in range(N):
            pos = lens[b] - n + i
            live = i < n and pos >= 0
            for w, h, out in zip(want, held, (ko, vo)):
                if live:
                    assert torch.equal(h[:, pos], w[:, i]), (b, i)
                    assert torch.equal(out.cpu()[b, :, i].double(), w[:, i]), (b, i)
                else:
                    assert (out[b, :, i] == 3.0).all(), (b, i)
            if live:
                r, pg = pos % page, int(tab[b, pos // page])
                e = torch.arange(d)
                for at in (r * (d // 2) + e // 2,
                           page * d // 2 + ((r // 64 * (d // 32) + e // 32) * 16 + r % 16) * 4 + r % 64 // 16,
                           page * (d // 2 + d // 32) + ((r // 4 * (d // 4) + e // 4) * 4 + r % 4) * 2 + e % 4 // 2,
                           page * (d + d // 32) + (((r // 64 * (d // 32) + e // 32) * 4 + r % 16 // 4) * 4 + r % 64 // 16) * 4 + r % 4):
                    touched[pg, :, at] = True
    # nothing but the rows' own bytes has changed
    assert torch.equal(host[~touched], before[~touched])


def test_extreme_values():
    import torch
    import paper_2606_07713_amd as moa
    cache, table = _pool(1, 64, 64, 1, 64, torch.Generator().manual_seed(1))
    x = torch.zeros((1, 1, 8, 64))
    x[0, 0, 0, 3] = math.inf
    x[0, 0, 1, 40] = math.nan
    x[0, 0, 2] = torch.finfo(torch.bfloat16).max
    x[0, 0, 3] = 2.0 ** -130
    x[0, 0, 4, ::2] = -7.0 * 2.0 ** -127
    x[0, 0, 5] = torch.linspace(-7, 7, 64)
    x[0, 0, 6] = -0.0
    x[0, 0, 7, 5] = -math.inf
    for dt in (torch.float32, torch.bfloat16):
        k = x.to(dt).to("cuda")
        moa.kv4_write(k, k, cache, _ints([8]), page_table=table)
        ko, vo = moa.kv4_read(cache, 8, 64, _ints([8]), page_table=table, out_dtype=torch.float32)
        want = quantised(k.cpu())
        for got in (ko, vo):
            assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got.cpu().double()), torch.nan_to_num(want))
            assert torch.isfinite(got[0, 0, 2:7]).all()


def test_tokens_outside_are_skipped():
    # positions behind the capacity and pages outside the pool: nothing is written, nothing read
    import torch
    import paper_2606_07713_amd as moa
    cache, _ = _pool(2, 64, 64, 2, 128, torch.Generator().manual_seed(1), fill=0x55)
    before = cache.clone()
    k = torch.randn((2, 2, 9, 128), device="cuda")
    table = _ints([[0, -1], [10 ** 9, 1]])
    # sequence 0: tokens 60 .. 68, of which 64.. lie on page -1; sequence 1: 120 .. 128 of capacity 128
    moa.kv4_write(k, k, cache, _ints([69, 129]), page_table=table)
    out = torch.full((2, 2, 9, 128), 3.0, device="cuda")
    vout = out.clone()
    moa.kv4_read(cache, 9, 128, _ints([69, 129]), page_table=table, k_out=out, v_out=vout)
    torch.cuda.synchronize()
    assert (out[0, :, 4:] == 3.0).all() and (out[1, :, 8] == 3.0).all()
    assert torch.equal(out[0, :, :4].cpu().double(), quantised(k[0, :, :4].cpu()))
    assert torch.equal(vout[1, :, :8].cpu().double(), quantised(k[1, :, :8].cpu()))
    assert torch.equal(cache[2:], before[2:])


def _attention(q, K, V, seen, scale):
    """fp64 (O, LSE, sum P|V|, max scale * sum |q k|) of one head: q [N, d], row i sees seen[i]."""
    import torch
    s = q @ K.t() * scale
    hide = torch.arange(K.shape[0])[None] >= seen[:, None]
    s = s.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(hide, 0.0, torch.exp(s - lse[:, None]))
    V0 = torch.where(torch.isnan(V), 0.0, V)
    o, mag = p @ V0, p @ V0.abs()
    nan = (~hide).double() @ torch.isnan(V).double() > 0
    o[nan] = math.nan
    empty = seen <= 0
    o[empty], mag[empty] = 0, 0
    reach = (q.abs() @ torch.nan_to_num(K).abs().t()).masked_fill(hide, 0).amax(-1) * abs(scale) if K.shape[0] else torch.zeros(q.shape[0])
    return o, lse, mag, reach


# B, Hq, Hk, N, d, page, lens, new_lens, causal, scale, splits, out
ATTNS = [
    (1, 1, 1, 1, 64, 64, [1], None, True, None, 0, "bf16"),
    (2, 4, 1, 1, 128, 64, [1, 65], None, True, None, 0, "f32"),
    (3, 8, 2, 1, 128, 128, [0, 63, 700], None, False, None, 0, "bf16"),
    (1, 32, 8, 1, 128, 64, [1030], None, True, None, 0, "bf16"),
    (2, 12, 4, 4, 64, 192, [4, 1000], None, True, None, 3, "bf16"),
    (2, 16, 1, 3, 128, 64, [2, 900], [3, 2], True, None, 0, "f32"),     # a query before token 0
    (1, 3, 3, 50, 64, 64, [130], None, True, None, 0, "f32"),
    (2, 4, 2, 70, 128, 128, [70, 400], [33, 70], True, 0.02, 0, "bf16"),
    (1, 8, 2, 37, 128, 256, [900], None, False, -0.1, 2, "f32"),
    (1, 2, 1, 20, 64, 64, [300], None, True, 0.0, 0, "f32"),
    (1, 20, 1, 1, 64, 64, [257], None, True, None, 256, "bf16"),
    (1, 6, 2, 200, 64, 64, [2300], None, True, None, 0, "bf16"),
]


def _cache_of(B, Hk, d, page, lens, seed=3, paged=True, std=1.0):
    """A cache that holds random tokens: (cache, table, max_pages * page)."""
    import torch
    import paper_2606_07713_amd as moa
    gen = torch.Generator().manual_seed(seed)
    cap = max(max(lens), 1)
    cache, table = _pool(B, cap, page, Hk, d, gen, paged)
    k, v = (torch.randn((B, Hk, cap, d), generator=gen).mul(std).to(torch.bfloat16).to("cuda") for _ in range(2))
    moa.kv4_write(k, v, cache, _ints(lens), page_table=table, new_lens=_ints(lens))
    return cache, table


def _check_attn(q, cache, table, page, lens, new, causal, scale, o, lse, poison=None):
    import torch
    B, Hq, N, d = q.shape
    Hk = cache.shape[1]
    host, tab = cache.cpu(), None if table is None else table.cpu()
    sc = scale if scale is not None else float(torch.tensor(1 / math.sqrt(d)).float())
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[o.dtype]
    worst = worst_l = 0.0
    for b in range(B):
        K, V = stored(host, page, d, tab, b, lens[b])
        n = N if new is None else new[b]
        at = torch.arange(n) + lens[b] - n + 1
        seen = at if causal else torch.full((n,), lens[b])
        for h in range(Hq):
            ref, l, mag, reach = _attention(q[b, h, :n].cpu().double(), K[h // (Hq // Hk)], V[h // (Hq // Hk)], seen, sc)
            got, gl = o[b, h, :n].cpu().double(), lse[b, h, :n].cpu().double()
            assert torch.equal(torch.isnan(got), torch.isnan(ref)), (b, h)
            ds = (d + 4) * U * reach
            sums = (lens[b] / 64 + 64) * U
            lim = (2.0 ** -8 + 2 * ds[:, None] + sums) * mag + half * ref.abs() + 1e-30
            err = torch.nan_to_num((got - ref).abs())
            worst = max(worst, (err / torch.nan_to_num(lim, nan=1.0)).max().item() if n else 0.0)
            empty = seen <= 0
            assert (gl[empty] == -math.inf).all()
            lerr = (gl - l)[~empty].abs() / (ds + sums + 4 * U * l.abs())[~empty]
            worst_l = max(worst_l, lerr.max().item() if lerr.numel() else 0.0)
    _say(f"  O worst {worst:.2f} of the bound, LSE {worst_l:.2f}")
    assert worst <= 1 and worst_l <= 1


@pytest.mark.parametrize("case", ATTNS, ids=lambda c: "x".join(map(str, c[:6])) + f"_{max(c[6])}_{'c' if c[8] else 'f'}")
def test_attention(case):
    import torch
    import paper_2606_07713_amd as moa
    B, Hq, Hk, N, d, page, lens, new, causal, scale, splits, odt = case
    _say(f"kv4 attention {case}")
    cache, table = _cache_of(B, Hk, d, page, lens)
    q = torch.randn((B, N, Hq, d), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to("cuda").transpose(1, 2)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[odt]
    out = torch.full((B, Hq, N, d), 3.0, dtype=dt, device="cuda")
    o, lse = moa.kv4_attn_fwd(q, cache, _ints(lens), page_table=table, new_lens=None if new is None else _ints(new),
                              causal=causal, scale=scale, num_splits=splits, out_dtype=dt, out=out, return_lse=True)
    torch.cuda.synchronize()
    _check_attn(q, cache, table, page, lens, new, causal, scale, o, lse)
    for b in range(B):
        if new is not None:
            assert (o[b, :, new[b]:] == 3.0).all()


def test_no_page_table_and_strided_output():
    import torch
    import paper_2606_07713_amd as moa
    lens = [100, 320]
    cache, table = _cache_of(2, 2, 128, 320, lens, paged=False)
    assert table is None
    q = torch.randn((2, 8, 2, 128), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to("cuda")
    out = torch.zeros((2, 2, 8, 128), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    o, lse = moa.kv4_attn_fwd(q, cache, _ints(lens), causal=True, out=out, return_lse=True)
    torch.cuda.synchronize()
    _check_attn(q, cache, None, 320, lens, None, True, None, o, lse)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,causal", [(1, True), (7, True), (40, True), (5, False)])
def test_nan_blocks_reach_only_the_rows_that_see_them(N, causal, d):
    # a token with a NaN in one value block, seen by some rows of the tile; unset memory behind
    import torch
    import paper_2606_07713_amd as moa
    lens = [150]
    cache, table = _cache_of(1, 1, d, 64, lens)
    for at, where in ((149, 40), (146, d - 28)):
        v = torch.zeros((1, 1, 1, d), device="cuda")
        v[..., where] = math.nan
        moa.kv4_write(torch.zeros_like(v), v, cache, _ints([at + 1]), page_table=table)
    q = torch.randn((1, 4, N, d), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to("cuda")
    for splits in (1, 2):
        o, lse = moa.kv4_attn_fwd(q, cache, _ints(lens), page_table=table, causal=causal, return_lse=True,
                                  out_dtype=torch.float32, num_splits=splits)
        torch.cuda.synchronize()
        _check_attn(q, cache, table, 64, lens, None, causal, None, o, lse)


def test_nan_key_makes_the_rows_that_see_it_nan():
    import torch
    import paper_2606_07713_amd as moa
    cache, table = _cache_of(1, 1, 64, 64, [80])
    k = torch.zeros((1, 1, 1, 64), device="cuda")
    k[..., 7] = math.inf
    moa.kv4_write(k, torch.zeros_like(k), cache, _ints([79]), page_table=table)
    q = torch.randn((1, 2, 4, 64), device="cuda").to(torch.bfloat16)
    for splits in (1, 2):
        o, lse = moa.kv4_attn_fwd(q, cache, _ints([80]), page_table=table, causal=True, return_lse=True, num_splits=splits)
        assert torch.isnan(o[:, :, 2:]).all() and torch.isnan(lse[:, :, 2:]).all()
        assert torch.isfinite(o[:, :, :2]).all() and torch.isfinite(lse[:, :, :2]).all()


def test_pages_outside_the_pool_hold_nothing():
    import torch
    import paper_2606_07713_amd as moa
    cache, table = _cache_of(1, 2, 64, 64, [256])
    q = torch.randn((1, 2, 1, 64), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to("cuda")
    k, v = moa.kv4_read(cache, 256, 64, _ints([256]), page_table=table, out_dtype=torch.float32)
    for bad in (-1, cache.shape[0], 2 ** 31 - 1):
        t = table.clone()
        t[0, 1] = bad
        o = moa.kv4_attn_fwd(q, cache, _ints([256]), page_table=t, causal=True, out_dtype=torch.float32)
        keep = [*range(64), *range(128, 256)]
        s = (q.float() * k[:, :, keep]).sum(-1) / 8.0
        want = (torch.softmax(s.double(), -1)[..., None] * v[:, :, keep].double()).sum(-2)
        # weights rounded to bf16, |V| <= 6
        assert (o[:, :, 0].double() - want).abs().max() < 6 * 2.0 ** -8
    empty = moa.kv4_attn_fwd(q, cache[:0], _ints([256]), page_table=table, causal=True)
    assert not empty.any()


def test_extreme_scores():
    # scores of several hundred, references raised again and again
    import torch
    import paper_2606_07713_amd as moa
    lens = [1500]
    cache, table = _cache_of(1, 2, 128, 64, lens, std=4.0)
    q = (8 * torch.randn((1, 4, 6, 128), generator=torch.Generator().manual_seed(2))).to(torch.bfloat16).to("cuda")
    for scale in (0.3, -0.3):
        o, lse = moa.kv4_attn_fwd(q, cache, _ints(lens), page_table=table, causal=True, scale=scale, return_lse=True)
        torch.cuda.synchronize()
        _check_attn(q, cache, table, 64, lens, None, True, scale, o, lse)


def test_no_and_almost_no_scale_against_huge_scores():
    # scores of 0 and +-2^126 times 0: equal weights; times 2^-130: weights exp(0), exp(+-2^-4)
    import torch
    import paper_2606_07713_amd as moa
    cache, table = _pool(1, 64, 64, 1, 64, torch.Generator().manual_seed(1))
    k = torch.zeros((1, 1, 40, 64), device="cuda")
    k[:, :, 1::3, 0], k[:, :, 2::3, 0] = 2.0 ** 63, -2.0 ** 63
    v = torch.arange(40, device="cuda").remainder(3).eq(1).float()[None, None, :, None].expand(1, 1, 40, 64).contiguous()
    moa.kv4_write(k, v, cache, _ints([40]), page_table=table)
    q = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0 ** 63
    for scale in (0.0, 2.0 ** -130, -2.0 ** -130):
        o = moa.kv4_attn_fwd(q, cache, _ints([40]), page_table=table, causal=True, scale=scale, out_dtype=torch.float32)
        for i, n in enumerate((39, 40)):
            w = torch.exp(k[0, 0, :n, 0].double() * 2.0 ** 63 * scale)
            want = (w * v[0, 0, :n, 0].double()).sum() / w.sum()
            # weights rounded to bf16 (2^-8 of each, in a mean of zeros and ones), the sums to fp32
            assert (o[0, 0, i].double() - want).abs().max() <= want * (2.0 ** -8 + 2.0 ** -18)


def test_norm_rope_write_attend_together():
    """A prompt, then decoded tokens, as a layer uses them: projections' heads normalised and
    rotated, keys and values written, queries attending; eagerly and replayed from a graph."""
    import torch
    import paper_2606_07713_amd as moa
    B, Hq, Hk, d, page, prompt = 2, 8, 2, 128, 64, 75
    gen = torch.Generator().manual_seed(6)
    cache, table = _pool(B, 128, page, Hk, d, gen)
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).to("cuda") for _ in range(2)]
    freq = (10000.0 ** (-torch.arange(d // 2) * 2 / d)).float().to("cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")

    def layer(x, pos, out):
        q, k, v = x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + Hk].transpose(1, 2), x[:, :, Hq + Hk:].transpose(1, 2)
        q, k = moa.qk_norm_rope(q, k, positions=pos, inv_freq=freq, q_weight=w[0], k_weight=w[1])
        moa.kv4_write(k, v, cache, lens, page_table=table)
        return (q, k, *moa.kv4_attn_fwd(q, cache, lens, page_table=table, causal=True, out=out, return_lse=True))

    def tokens(n):
        return torch.randn((B, n, Hq + 2 * Hk, d), generator=gen).to(torch.bfloat16).to("cuda")

    lens.fill_(prompt)
    out = torch.empty((B, prompt, Hq, d), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    q, k, o, lse = layer(tokens(prompt), torch.arange(prompt, device="cuda").expand(B, prompt).contiguous(), out)
    torch.cuda.synchronize()
    _check_attn(q, cache, table, page, [prompt] * B, None, True, None, o, lse)

    x, pos = tokens(1), torch.empty((B, 1), dtype=torch.int64, device="cuda")
    out1 = torch.empty((B, Hq, 1, d), dtype=torch.bfloat16, device="cuda")
    lens.fill_(prompt + 1)
    pos.fill_(prompt)
    layer(x, pos, out1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, k, o, lse = layer(x, pos, out1)
    for step in range(4):
        x.copy_(tokens(1))
        lens.fill_(prompt + 1 + step)
        pos.fill_(prompt + step)
        graph.replay()
        torch.cuda.synchronize()
        _check_attn(q, cache, table, page, [prompt + 1 + step] * B, None, True, None, o, lse)
        got = o.clone()
        assert torch.equal(layer(x, pos, torch.empty_like(out1))[2], got)


def test_pool_beyond_four_gigabytes():
    # pages whose offsets pass 32 bits; most of the pool is never touched
    import torch
    import paper_2606_07713_amd as moa
    page, Hk, d = 256, 8, 128
    num = (5 << 30) // (Hk * page * (d + d // 16))
    cache = moa.kv4_cache(num, Hk, page, d)
    table = _ints([[num - 1, 0, num // 2]])
    lens, gen = [600], torch.Generator().manual_seed(3)
    k, v = (torch.randn((1, Hk, 600, d), generator=gen).to(torch.bfloat16).to("cuda") for _ in range(2))
    moa.kv4_write(k, v, cache, _ints(lens), page_table=table)
    ko, vo = moa.kv4_read(cache, 600, d, _ints(lens), page_table=table)
    for got, x in ((ko, k), (vo, v)):
        assert torch.equal(got.cpu().double(), quantised(x.cpu()))
    q = torch.randn((1, 16, 2, d), generator=gen).to(torch.bfloat16).to("cuda")
    o, lse = moa.kv4_attn_fwd(q, cache, _ints(lens), page_table=table, causal=True, return_lse=True)
    torch.cuda.synchronize()
    near = cache[[num - 1, 0, num // 2]]
    _check_attn(q, near, _ints([[0, 1, 2]]), page, lens, None, True, None, o, lse)


def test_given_stream_owns_what_the_call_allocates():
    # calls on a stream of their own, while the current stream allocates and writes
    import torch
    import paper_2606_07713_amd as moa
    lens = [3000]
    cache, table = _cache_of(1, 2, 128, 64, lens)
    q = torch.randn((1, 8, 1, 128), device="cuda").to(torch.bfloat16)
    seq = _ints(lens)
    want = moa.kv4_attn_fwd(q, cache, seq, page_table=table)
    assert moa.moa_kv4_attn_num_splits(1, 8, 2, 1, 128, 64, table.shape[1], 0, 0) > 1
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(20):
        got.append(moa.kv4_attn_fwd(q, cache, seq, page_table=table, stream=s))
        torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_on_another_stream():
    import torch
    import paper_2606_07713_amd as moa
    lens = [500]
    cache, table = _cache_of(1, 2, 128, 64, lens)
    q = torch.randn((1, 8, 1, 128), device="cuda").to(torch.bfloat16)
    want = moa.kv4_attn_fwd(q, cache, _ints(lens), page_table=table)
    s = torch.cuda.Stream()
    seq = _ints(lens)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = moa.kv4_attn_fwd(q, cache, seq, page_table=table)
    b = moa.kv4_attn_fwd(q, cache, seq, page_table=table, stream=s, out=torch.empty_like(a),
                         workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
