"""Attention in a window (``win_attn_fwd``) against its definition in fp64."""
import math

import pytest
import torch

from win_util import Exact, close, close_lse, visible

pytestmark = pytest.mark.gpu


def _normal(seed, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).cuda()


def _exact(q, k, v, left, right, sinks, scale=None, do=None):
    B, Nq, Nk = q.shape[0], q.shape[2], k.shape[2]
    pos = torch.arange(Nk - Nq, Nk, device="cuda").expand(B, Nq)
    see = visible(pos, Nk, torch.full((B,), Nk, device="cuda"), left, right, sinks)
    return Exact(q, k, v, see, 1 / math.sqrt(q.shape[3]) if scale is None else scale, do)


def _check(q, k, v, left=-1, right=-1, sinks=0, scale=None, num_splits=0, dtypes=(torch.bfloat16, torch.float32)):
    import paper_2606_07713_amd as moa
    x = _exact(q, k, v, left, right, sinks, scale)
    B, Hq, Nq, d = q.shape
    for dt in dtypes:
        o, lse = moa.win_attn_fwd(q, k, v, left, right, sinks, scale=scale, out_dtype=dt, return_lse=True,
                                  num_splits=num_splits)
        torch.cuda.synchronize()
        terms = 3 if dt is torch.float32 else 1 if Nq * (Hq // k.shape[1]) > 32 else 2
        close(o, x.o, x.o_bound(dt, terms), x.odd)
        close_lse(lse, x.lse, x.lse_bound(), x.odd.any(-1))


WINDOWS = [(-1, -1, 0), (-1, 0, 0), (0, 0, 0), (7, 0, 0), (100, 0, 4), (31, 17, 0), (64, 64, 3), (5, -1, 70), (-1, 3, 0)]


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Nk,G", [(1, 1, 1), (1, 300, 4), (3, 2, 2), (5, 33, 6), (17, 64, 1), (200, 200, 1), (130, 333, 3),
                                     (65, 40, 2), (129, 129, 5)])
def test_sizes(window, d, Nq, Nk, G):
    Hk = 2
    q, k, v = _normal(1, 2, Hk * G, Nq, d), _normal(2, 2, Hk, Nk, d), _normal(3, 2, Hk, Nk, d)
    _check(q, k, v, *window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("splits", [1, 2, 3, 17, 256])
@pytest.mark.parametrize("Nq,G", [(1, 4), (4, 6), (70, 3)])
def test_splits(d, splits, Nq, G):
    q, k, v = _normal(4, 1, 2 * G, Nq, d), _normal(5, 1, 2, 1000, d), _normal(6, 1, 2, 1000, d)
    for window in ((-1, 0, 0), (200, 0, 5)):
        _check(q, k, v, *window, num_splits=splits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [2, 90])
def test_strided_views(d, Nq):
    """Slices of a packed projection output [B, N, Hq + 2 Hk, d], out and back."""
    import paper_2606_07713_amd as moa
    B, Hq, Hk, N = 2, 6, 2, 150
    x = _normal(7, B, N, Hq + 2 * Hk, d).transpose(1, 2)
    q, k, v = x[:, :Hq, N - Nq:], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    _check(q, k, v, 40, 0, 2)
    out = torch.full((B, Nq, Hq, 2 * d), 7.0, dtype=torch.bfloat16, device="cuda")
    o = moa.win_attn_fwd(q, k, v, 40, 0, 2, out=out[..., :d].transpose(1, 2))
    assert torch.equal(o, moa.win_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), 40, 0, 2))
    assert bool((out[..., d:] == 7).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("splits", [1, 2, 16])
@pytest.mark.parametrize("Nq,G", [(1, 2), (20, 1), (90, 2)])
def test_values_near_the_largest(Nq, G, splits, d):
    """Sums of such values leave fp32 before they are divided, in a split and in the join of splits."""
    v = _normal(50, 1, 2, 1024, d)
    v = (torch.where(v < 0, -1.0, 1.0) * 3e38 - v.float() * 1e36).to(torch.bfloat16)
    v[..., d // 2:] = 3e38
    _check(_normal(51, 1, 2 * G, Nq, d), _normal(52, 1, 2, 1024, d), v, -1, -1, 0, num_splits=splits)
    _check(_normal(51, 1, 2 * G, Nq, d), _normal(52, 1, 2, 1024, d), v, 300, 0, 0, num_splits=splits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rise", [100.0, 119.5, 126.0, 127.5, 140.0])
@pytest.mark.parametrize("Nq,G", [(1, 2), (20, 1), (90, 2)])
def test_scores_that_rise_in_every_split(Nq, G, rise, d):
    """One key of every 64 stands so many log2 units above the others: a split's sum is the largest
    number or near it, and 16 of them are added."""
    q, k, v = _normal(53, 1, 2 * G, Nq, d), _normal(54, 1, 2, 1024, d), _normal(55, 1, 2, 1024, d)
    q[..., 0], k[..., 0] = 1.0, 0.0
    q[..., 1:], k[:, :, 60::64, 0] = 0.0, 1.0
    _check(q, k, v, -1, -1, 0, scale=rise * math.log(2), num_splits=16)
    _check(q, k, v, -1, -1, 0, scale=rise * math.log(2), num_splits=1)


@pytest.mark.parametrize("d", [64, 128])
def test_many_workgroups(d):
    """More than two workgroups for every compute unit: other tiles are taken at d = 128."""
    q, k, v = _normal(21, 40, 16, 70, d), _normal(22, 40, 8, 150, d), _normal(23, 40, 8, 150, d)
    k[3, 2, 100], v[5, 1, 149, 4], v[39, 7, 81] = math.nan, math.inf, math.nan
    for window in ((-1, 0, 0), (45, 0, 3), (20, 9, 40)):
        _check(q, k, v, *window)


@pytest.mark.parametrize("Nq", [3, 100])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0, 1e-42])
def test_scales(Nq, scale):
    q, k, v = _normal(8, 1, 4, Nq, 64), _normal(9, 1, 2, 120, 64), _normal(10, 1, 2, 120, 64)
    _check(q, k, v, 50, 0, 1, scale=scale)


@pytest.mark.parametrize("Nq,splits", [(4, 1), (4, 3), (100, 1), (100, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_has_no_part(Nq, splits, d, what):
    """NaN and infinities in keys and values of the windows' middle: only rows that see them know."""
    import paper_2606_07713_amd as moa
    q, k, v = _normal(11, 2, 4, Nq, d), _normal(12, 2, 2, 200, d), _normal(13, 2, 2, 200, d)
    k[0, 1, 150], v[0, 0, 198, 5], v[1, 1, 60], k[1, 0, 0, 3], v[1, 0, 199, 0] = what, what, what, what, what
    for window in ((10, 0, 0), (60, 0, 3), (-1, 0, 0)):
        _check(q, k, v, *window, num_splits=splits)
        x = _exact(q, k, v, *window)
        o = moa.win_attn_fwd(q, k, v, *window, num_splits=splits)
        v_bad = x.odd & ~x.p.isnan().any(-1, keepdim=True)     # a value's own infinity or NaN, with its weight
        assert not bool((o.isfinite() & v_bad).any())


@pytest.mark.parametrize("Nq", [2, 100])
def test_large_values_and_scores(Nq):
    """Values up to the largest, and scores beyond fp32: the definition's results."""
    q, k, v = _normal(14, 1, 2, Nq, 64), _normal(15, 1, 1, 130, 64), _normal(16, 1, 1, 130, 64)
    v = (v.float().sign() * 3.3e38).to(torch.bfloat16)
    _check(q, k, v, 90, 0, 2, dtypes=(torch.float32,))
    import paper_2606_07713_amd as moa
    big = (q.float() * 1e25).to(torch.bfloat16), (k.float() * 1e25).to(torch.bfloat16)
    v = _normal(17, 1, 1, 130, 64)
    o = moa.win_attn_fwd(*big, v, -1, 0, out_dtype=torch.float32)
    s = torch.where(torch.arange(130, device="cuda") <= torch.arange(130 - Nq, 130, device="cuda")[:, None],
                    big[0].double() @ big[1].double().transpose(2, 3), -math.inf)
    want = v[0, 0][s.argmax(-1)].float()           # one key has all the weight
    assert torch.allclose(o, want, rtol=0, atol=0)


@pytest.mark.parametrize("Nq", [4, 100])
@pytest.mark.parametrize("rise", [60, 120, 200, 2000])
def test_scores_that_rise(Nq, rise):
    """Keys whose scores grow from the first to the last: the reference stays that of the first ones."""
    q = _normal(24, 1, 2, Nq, 64)
    q[..., 0] = 8
    k, v = _normal(25, 1, 2, 400, 64), _normal(26, 1, 2, 400, 64)
    k[..., 0] = torch.linspace(0, rise, 400, device="cuda").to(torch.bfloat16)   # scores up to `rise` higher
    for splits in (1, 3):
        _check(q, k, v, -1, 0, 0, num_splits=splits)
        _check(q, k, v, 250, 0, 4, num_splits=splits)


def test_nothing_to_do():
    import paper_2606_07713_amd as moa
    for B, Hq, Nq, Nk in ((0, 2, 3, 4), (1, 0, 3, 4), (1, 2, 0, 4), (2, 2, 3, 0), (1, 2, 60, 0)):
        q, k = _normal(1, B, Hq, Nq, 64), _normal(2, B, 1, Nk, 64)
        o, lse = moa.win_attn_fwd(q, k, k, 3, 0, return_lse=True)
        assert o.shape == q.shape and bool((o == 0).all()) and bool((lse == -math.inf).all())


def test_another_stream_and_the_same_bits():
    import paper_2606_07713_amd as moa
    q, k, v = _normal(18, 2, 8, 500, 128), _normal(19, 2, 2, 500, 128), _normal(20, 2, 2, 500, 128)
    want = moa.win_attn_fwd(q, k, v, 99, 0, 4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = moa.win_attn_fwd(q, k, v, 99, 0, 4, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    ws = torch.full((moa.moa_win_attn_workspace_bytes(2, 8, 2, 500, 500, 128, 99, 0, 4, 3),), 255, dtype=torch.uint8, device="cuda")
    a = moa.win_attn_fwd(q, k, v, 99, 0, 4, num_splits=3, workspace=ws)
    assert torch.equal(a, moa.win_attn_fwd(q, k, v, 99, 0, 4, num_splits=3))
