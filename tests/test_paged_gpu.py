"""The paged bf16 cache: appending (``paged_append``) and the attention over it
(``paged_attn_fwd``) against their definitions in fp64."""
import math

import pytest
import torch

from win_util import EPS, Exact, close, close_lse, visible

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _normal(seed, *shape, std=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """Pools of random pages, every sequence's pages in no order."""

    def __init__(self, lens, Hk, page, d, layout="apart", seed=0, spare=2, fill=None):
        self.lens, self.page, self.d, self.Hk = lens, page, d, Hk
        pages = [-(-max(n, 0) // page) for n in lens]
        total = sum(pages) + spare
        order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
        most = max(pages) + 1
        self.table = torch.full((len(lens), most), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.table = self.table.cuda()
        if layout == "apart":
            self.k, self.v = _normal(seed + 1, total, Hk, page, d), _normal(seed + 2, total, Hk, page, d)
        elif layout == "pages":        # keys and values of a page next to each other
            x = _normal(seed + 1, total, 2, Hk, page, d)
            self.k, self.v = x[:, 0], x[:, 1]
        else:                          # tokens first
            x = _normal(seed + 1, total, page, 2 * Hk, d).transpose(1, 2)
            self.k, self.v = x[:, :Hk], x[:, Hk:]
        if fill is not None:
            self.k.fill_(fill)
            self.v.fill_(fill)

    def rows(self, pool, b, n):
        """Tokens 0 .. n - 1 of sequence b: [Hk, n, d]; NaN where there is no page."""
        j = torch.arange(n, device="cuda")
        page = self.table[b].long()[(j // self.page).clamp(max=self.table.shape[1] - 1)]
        has = (j // self.page < self.table.shape[1]) & (page >= 0) & (page < pool.shape[0])
        x = pool[torch.where(has, page, 0), :, j % self.page].transpose(0, 1).double()
        return torch.where(has[None, :, None], x, math.nan), has


def _check(c, q, left=-1, right=-1, sinks=0, new=None, num_splits=0, dtypes=(BF16, torch.float32), **kw):
    import paper_2606_07713_amd as moa
    B, Hq, N, d = q.shape
    new_lens = None if new is None else _i32(new)
    for dt in dtypes:
        out = torch.full((B, Hq, N, d), 7.0, dtype=dt, device="cuda")
        o, lse = moa.paged_attn_fwd(q, c.k, c.v, _i32(c.lens), page_table=c.table, new_lens=new_lens, left=left, right=right,
                                    sinks=sinks, out_dtype=dt, return_lse=True, num_splits=num_splits, out=out, **kw)
        torch.cuda.synchronize()
        terms = 3 if dt is torch.float32 else 1 if N * (Hq // c.Hk) > 32 else 2
        for b, n in enumerate(c.lens):
            real = N if new is None else min(max(new[b], 0), N)
            assert bool((o[b, :, real:] == 7).all())
            if not real:
                continue
            m = max(n, 1)
            (k, has), (v, _) = c.rows(c.k, b, m), c.rows(c.v, b, m)
            pos = torch.arange(n - real, n, device="cuda")[None]
            see = visible(pos, m, torch.tensor([n], device="cuda"), left, right, sinks) & has
            x = Exact(q[b:b + 1, :, :real], k[None], v[None], see, 1 / math.sqrt(d))
            close(o[b:b + 1, :, :real], x.o, x.o_bound(dt, terms), x.odd)
            close_lse(lse[b:b + 1, :, :real], x.lse, x.lse_bound(), x.odd.any(-1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("N,G", [(1, 1), (1, 4), (1, 24), (4, 3), (5, 6), (33, 4), (150, 1)])
@pytest.mark.parametrize("window", [(-1, 0, 0), (-1, -1, 0), (37, 0, 5), (200, 10, 100)], ids=str)
def test_attention(d, page, N, G, window):
    lens = [N, 401, 64 + N, 1 + N]
    c = Cache(lens, 2, page, d)
    _check(c, _normal(9, len(lens), 2 * G, N, d, std=1.5), *window)


@pytest.mark.parametrize("splits", [1, 2, 5, 32])
@pytest.mark.parametrize("N", [1, 3, 40])
def test_splits_of_ragged_lengths(splits, N):
    c = Cache([700, N, 1500, 130 + N, 0], 3, 16, 64)
    for window in ((-1, 0, 0), (300, 0, 4)):
        _check(c, _normal(9, 5, 6, N, 64), *window, num_splits=splits, max_len=1500)


@pytest.mark.parametrize("page", [16, 64])
def test_many_workgroups(page):
    """More than two workgroups for every compute unit, pages that are not there among them."""
    lens = [40 + 13 * i % 200 for i in range(80)]
    c = Cache(lens, 8, page, 128)
    c.table[7, 0] = -1
    c.table[60:, 1] = -1
    _check(c, _normal(9, 80, 16, 40, 128), 70, 0, 3, dtypes=(BF16,))


@pytest.mark.parametrize("layout", ["pages", "tokens"])
@pytest.mark.parametrize("N", [2, 50])
def test_layouts_of_the_pools(layout, N):
    c = Cache([300, 77 + N], 2, 32, 128, layout)
    _check(c, _normal(9, 2, 8, N, 128).transpose(1, 2).contiguous().transpose(1, 2), 100, 0, 3)


@pytest.mark.parametrize("N", [1, 4, 40])
def test_fewer_new_tokens_than_rows(N):
    c = Cache([200, 90, 60, 41], 2, 16, 64)
    _check(c, _normal(9, 4, 4, N, 64), -1, 0, 0, new=[N, 0, max(1, N // 2), N + 5])
    _check(c, _normal(9, 4, 4, N, 64), 30, 0, 1, new=[1, -3, N, 1], num_splits=3)


@pytest.mark.parametrize("N", [1, 4, 40])
@pytest.mark.parametrize("splits", [1, 3])
def test_pages_that_are_not_there(N, splits):
    """Entries outside the pool, lengths behind the capacity, sequences shorter than their new tokens."""
    c = Cache([300, 280, 100, 5], 2, 16, 64)
    c.table[0, 3] = -1
    c.table[0, 10:12] = c.k.shape[0]
    c.table[1, :] = -5
    c.lens = [300, 280, c.table.shape[1] * 16 + 9, 3]
    _check(c, _normal(9, 4, 4, N, 64), -1, 0, 0, num_splits=splits)
    _check(c, _normal(9, 4, 4, N, 64), 90, 0, 20, num_splits=splits)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("N", [1, 3, 70])
def test_unset_memory_behind_the_tokens(d, page, N):
    """NaN in everything that holds no token of the sequence."""
    lens = [N, 130, 67 + N]
    c = Cache(lens, 2, page, d, fill=math.nan)
    g = torch.Generator().manual_seed(1)
    for b, n in enumerate(lens):
        for j in range(n):
            p = int(c.table[b, j // page])
            for pool in (c.k, c.v):
                pool[p, :, j % page] = torch.randn((2, d), generator=g).to(BF16).cuda()
    for splits in (1, 2):
        _check(c, _normal(9, 3, 8, N, d), -1, 0, 0, num_splits=splits)
        _check(c, _normal(9, 3, 8, N, d), -1, -1, 0, num_splits=splits)


def test_without_a_table():
    import paper_2606_07713_amd as moa
    k, v, q = _normal(1, 3, 2, 512, 64), _normal(2, 3, 2, 512, 64), _normal(3, 2, 4, 3, 64)
    lens = _i32([512, 100])
    got = moa.paged_attn_fwd(q, k, v, lens, right=0, left=50)
    for b, n in enumerate((512, 100)):
        want = moa.win_attn_fwd(q[b:b + 1], k[b:b + 1, :, :n], v[b:b + 1, :, :n], 50, 0)
        assert torch.equal(got[b:b + 1], want)


def test_far_pages():
    """A pool of more than 2^32 elements and bytes: pages at its end."""
    import paper_2606_07713_amd as moa
    k = torch.zeros((9000, 8, 512, 128), dtype=BF16, device="cuda")
    v = torch.zeros((9000, 8, 512, 128), dtype=BF16, device="cuda")
    c = Cache([1000], 8, 512, 128, spare=0)
    c.k, c.v = k, v
    c.table[0, :2] = _i32([8999, 8000])
    for p in (8999, 8000):
        k[p], v[p] = _normal(p, 8, 512, 128), _normal(p + 1, 8, 512, 128)
    for N in (1, 20):
        _check(c, _normal(3, 1, 16, N, 128), 700, 0, 2)
    q = _normal(4, 1, 8, 10, 128)
    moa.paged_append(None, q * 0 + 3, q * 0 + 5, k, v, _i32([1000]), page_table=c.table)
    assert bool((c.rows(k, 0, 1000)[0][:, 990:] == 3).all()) and bool((c.rows(v, 0, 1000)[0][:, 990:] == 5).all())


# ---- appending ------------------------------------------------------------------------------------


def _turned(x, w, pos, freq, eps, interleaved):
    """x [H, n, d] in fp64 normed and turned, and the size of each result's terms."""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    size = x.abs().clone()
    if freq is not None:
        r = 2 * freq.shape[0]
        a = pos.double()[:, None] * freq.double()
        cos, sin = a.cos(), a.sin()
        i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
        u, v = x[..., i].clone(), x[..., j].clone()
        x[..., i], x[..., j] = u * cos - v * sin, v * cos + u * sin
        size[..., i] = size[..., j] = u.abs() + v.abs()
    return x, size


def _check_append(c, q, k, v, new=None, positions=None, freq=None, wq=None, wk=None, interleaved=False, in_place=False,
                  q_out=None):
    import paper_2606_07713_amd as moa
    B, Hk, N, d = k.shape
    was = [c.k.clone(), c.v.clone()]
    q0, k0, v0 = (None if t is None else t.clone() for t in (q, k, v))
    if q is not None and q_out is None:
        q_out = q if in_place else torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    rest = None if q is None else q_out.clone()
    got = moa.paged_append(q, k, v, c.k, c.v, _i32(c.lens), page_table=c.table, new_lens=None if new is None else _i32(new),
                           positions=positions, inv_freq=freq, q_weight=wq, k_weight=wk, interleaved=interleaved, q_out=q_out)
    torch.cuda.synchronize()
    assert got is q_out
    kp, vp = was[0], was[1]
    touched = torch.zeros(kp.shape[:3], dtype=torch.bool, device="cuda")
    cap = c.table.shape[1] * c.page

    def near(got, x, w, at):
        want, size = _turned(x, w, at, freq, 1e-6, interleaved)
        # angle in fp32 turns (2^-23), sine and cosine, rsqrt and the mean (2^-20 together), one rounding
        close(got, want, want.abs() * EPS[BF16] + size * 2.0 ** -19 + 1e-30)

    for b, n in enumerate(c.lens):
        real = N if new is None else min(max(new[b], 0), N)
        at = torch.arange(n - real, n, device="cuda")
        pos = at if positions is None else positions[b, :real]
        if q is not None:
            near(q_out[b, :, :real], q0[b, :, :real], wq, pos)
            assert torch.equal(q_out[b, :, real:], rest[b, :, real:])
        for i in range(real):
            t = int(at[i])
            page = int(c.table[b, t // c.page]) if 0 <= t < cap else -1
            if not 0 <= page < kp.shape[0]:
                continue
            touched[page, :, t % c.page] = True
            kp[page, :, t % c.page] = c.k[page, :, t % c.page]       # checked here, below: all else as it was
            near(c.k[page, :, t % c.page][:, None], k0[b, :, i:i + 1], wk, pos[i:i + 1])
            assert torch.equal(c.v[page, :, t % c.page], v0[b, :, i].to(BF16))
            vp[page, :, t % c.page] = c.v[page, :, t % c.page]
    assert torch.equal(c.k, kp) and torch.equal(c.v, vp)


def _freq(r):
    return (10000.0 ** (-torch.arange(r // 2, dtype=torch.float64) * 2 / r)).float().cuda()


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,Hq,Hk,page", [(1, 4, 2, 16), (7, 6, 1, 32), (40, 2, 3, 16)])
@pytest.mark.parametrize("how", ["plain", "norm", "pairs", "values"])
def test_append(dtype, d, N, Hq, Hk, page, how):
    c = Cache([N, 100 + N, 33 + N], Hk, page, d)
    B = 3
    q, k, v = (_normal(s, B, h, N, d, std=2.0, dtype=dtype) for s, h in ((1, Hq), (2, Hk), (3, Hk)))
    wq, wk = (_normal(s, d, dtype=dtype) + 1 for s in (4, 5)) if how == "norm" else (None, None)
    freq = None if how == "values" else _freq(d if how != "pairs" else d // 2)
    _check_append(c, q, k, v, freq=freq, wq=wq, wk=wk, interleaved=how == "pairs")


@pytest.mark.parametrize("layout", ["pages", "tokens"])
def test_append_packed_and_in_place(layout):
    """q, k, v: slices of one projection output, the queries turned where they stand."""
    c = Cache([90, 64], 2, 32, 128, layout)
    x = _normal(1, 2, 20, 8 + 4, 128).transpose(1, 2)
    _check_append(c, x[:, :8], x[:, 8:10], x[:, 10:], freq=_freq(128), in_place=True)
    x = _normal(2, 2, 20, 8 + 4, 128).transpose(1, 2)
    _check_append(c, x[:, :8], x[:, 8:10], x[:, 10:], freq=_freq(64), wk=_normal(3, 128))


def test_append_skips():
    """Fewer tokens than rows, tokens before 0, behind the capacity and on pages outside the pool; and
    given positions, far ones."""
    c = Cache([60, 200, 100, 0], 2, 16, 64)
    c.table[1, 12] = -1
    c.table[0, 2] = c.k.shape[0]
    c.lens = [60, 200, c.table.shape[1] * 16 + 4, 3]
    q, k, v = _normal(1, 4, 4, 20, 64), _normal(2, 4, 2, 20, 64), _normal(3, 4, 2, 20, 64)
    pos = (torch.arange(4)[:, None] * 10 ** 9 + torch.arange(20)).cuda()
    for positions in (None, pos):
        _check_append(c, q, k, v, freq=_freq(64), positions=positions)
        _check_append(c, q, k, v, new=[20, 0, 7, 99], freq=_freq(32), positions=positions)
        _check_append(c, None, k, v, new=[-1, 5, 1, 2], freq=_freq(64), positions=positions)


def test_append_tiny_and_huge_rows():
    c = Cache([40], 1, 16, 64)
    k = _normal(1, 1, 1, 8, 64, dtype=torch.float32)
    k[0, 0, 1] *= 1e-30
    k[0, 0, 2] *= 1e30
    k[0, 0, 5] = 0
    _check_append(c, k * 1e-3, k, k, wq=torch.ones(64, device="cuda"), wk=_normal(2, 64, dtype=torch.float32), freq=_freq(64))
    # a value next to an infinite one stays as it is
    v = _normal(3, 1, 1, 8, 64)
    v[0, 0, 3, 7] = math.inf
    _check_append(c, None, _normal(4, 1, 1, 8, 64), v, freq=_freq(64))


# ---- together ---------------------------------------------------------------------------------------


@pytest.mark.parametrize("left,sinks", [(-1, 0), (100, 4)])
def test_a_prompt_then_steps_in_a_graph(left, sinks):
    """A prompt in two chunks, then single tokens by one captured graph: every step equals the whole
    sequence's attention computed at once."""
    import paper_2606_07713_amd as moa
    B, Hq, Hk, d, page, total, first = 2, 8, 2, 64, 16, 330, 300
    freq, wk = _freq(d), _normal(5, d) + 1
    x = _normal(1, B, total, Hq + 2 * Hk, d).transpose(1, 2)
    pool = moa.paged_cache(100, Hk, page, d)
    for t in pool:
        t.fill_(math.nan)
    table = torch.randperm(100, generator=torch.Generator().manual_seed(1))[: B * 22].int().view(B, 22).cuda()
    lens, new = _i32([0, 0]), None

    def step(rows, lens):
        q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:]
        q = moa.paged_append(q, k, v, *pool, lens, page_table=table, inv_freq=freq, k_weight=wk)
        return moa.paged_attn_fwd(q, *pool, lens, page_table=table, left=left, right=0, sinks=sinks)

    outs = []
    for a, b in ((0, 180), (180, first)):
        lens.fill_(b)
        outs.append(step(x[:, :, a:b], lens))
    token = x[:, :, :1].transpose(1, 2).contiguous().transpose(1, 2)
    lens.fill_(first + 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token.copy_(x[:, :, first:first + 1])
        step(token, lens)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(token, lens)
    for t in range(first, total):
        token.copy_(x[:, :, t:t + 1])
        lens.fill_(t + 1)
        graph.replay()
        torch.cuda.synchronize()
        outs.append(got.clone())
    q, k = moa.qk_norm_rope(x[:, :Hq], x[:, Hq:Hq + Hk], inv_freq=freq, k_weight=wk)
    v = x[:, Hq + Hk:]
    pos = torch.arange(total, device="cuda").expand(B, total)
    e = Exact(q, k, v, visible(pos, total, torch.full((B,), total, device="cuda"), left, 0, sinks), 1 / math.sqrt(d))
    close(torch.cat(outs, 2), e.o, e.o_bound(BF16, 1))
