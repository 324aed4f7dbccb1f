"""Attention in a window: rows that are done by the definition, and what LSE says of them and of the rows
beside them, against the definition in fp64."""
import math

import pytest
import torch

from test_window_gpu import _exact, _normal
from test_window_joins_gpu import close_lse
from win_util import close

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _check(q, k, v, left=-1, right=-1, sinks=0, num_splits=0):
    """O where a value is expected, LSE of every row."""
    import paper_2606_07713_amd as moa
    x = _exact(q, k, v, left, right, sinks)
    many = q.shape[2] * (q.shape[1] // k.shape[1]) > 32
    for dt in (BF16, torch.float32):
        o, lse = moa.win_attn_fwd(q, k, v, left, right, sinks, out_dtype=dt, return_lse=True, num_splits=num_splits)
        torch.cuda.synchronize()
        close(o, x.o, x.o_bound(dt, 3 if dt is torch.float32 else 1 if many else 2), x.odd)
        close_lse(lse, x.lse, x.lse_bound())
    return x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [3, 100])
@pytest.mark.parametrize("splits", [1, 2, 5])
@pytest.mark.parametrize("first,end", [(0, 64), (0, 32), (0, 130), (70, 71), (128, 192), (0, 300)])
def test_a_score_that_is_no_number(first, end, splits, Nq, d):
    """All keys that a row sees first, or some later ones, are NaN: LSE is too, whatever comes after them."""
    q, k, v = _normal(1, 2, 4, Nq, d), _normal(2, 2, 2, 300, d), _normal(3, 2, 2, 300, d)
    k[0, 1, first:end] = math.nan
    for window in ((-1, -1, 0), (-1, 0, 0), (80, 0, 2)):
        x = _check(q, k, v, *window, num_splits=splits)
        assert not bool(x.lse[0, :2].isnan().any())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [5, 100])
@pytest.mark.parametrize("splits", [1, 2])
def test_values_have_no_part_in_log_sums(splits, Nq, d):
    q, k, v = _normal(4, 2, 4, Nq, d), _normal(5, 2, 2, 200, d), _normal(6, 2, 2, 200, d)
    v[0, 0], v[1, 1, 60:150, 3], v[1, 0, 199] = math.nan, math.inf, -math.inf
    for window in ((-1, -1, 0), (-1, 0, 0), (30, 0, 3)):
        x = _check(q, k, v, *window, num_splits=splits)
        assert bool(x.lse.isfinite().all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("Nq,Nk", [(8, 3), (150, 70), (150, 1)])
def test_rows_that_see_nothing_beside_odd_ones(Nq, Nk, splits, d):
    """Causal queries before the first key, NaN in keys and values and in the queries themselves."""
    import paper_2606_07713_amd as moa
    q, k, v = _normal(7, 1, 4, Nq, d), _normal(8, 1, 2, Nk, d), _normal(9, 1, 2, Nk, d)
    k[0, 0, :2], v[0, 1, :1] = math.nan, math.nan
    for bad_queries in (False, True):
        if bad_queries:
            q[0, 0, ::3] = math.nan
        x = _check(q, k, v, -1, 0, 0, num_splits=splits)
        empty = Nq - Nk
        o, lse = moa.win_attn_fwd(q, k, v, -1, 0, return_lse=True, num_splits=splits)
        assert bool((x.lse[:, :, :empty] == -math.inf).all()) and bool((lse[:, :, :empty] == -math.inf).all())
        assert bool((o[:, :, :empty] == 0).all())


def _by_scores(q, k, v, scale, splits):
    """Where a score's fp32 products and sum are exact, only the weights' exponentials (2^-22), their
    arguments (fp32 numbers below 128, of scores in fp64: 2^-18 and |score| 2^-51), sums and products are off."""
    import paper_2606_07713_amd as moa
    s = q.double() @ k.double().repeat_interleave(q.shape[1] // k.shape[1], 1).transpose(2, 3) * scale
    v = v.double().repeat_interleave(q.shape[1] // v.shape[1], 1)
    p, lse = torch.softmax(s, -1), torch.logsumexp(s, -1)
    top = float(torch.where(s.isfinite(), s, 0.0).abs().max())
    o, got = moa.win_attn_fwd(q, k, v.to(BF16)[:, ::q.shape[1] // k.shape[1]], scale=scale, out_dtype=torch.float32, return_lse=True,
                              num_splits=splits)
    torch.cuda.synchronize()
    close(o, p @ v, (p @ v.abs()) * (2.0 ** -17 + top * 2.0 ** -51) + 1e-30)
    close(got, lse, lse.abs() * 2.0 ** -21 + 2.0 ** -17)


def _one_score(S, sign, Nq, Nk, d, seed):
    """Keys with scores of sign * 2 S, and q for scores of up to S and small steps beside it."""
    q, k, v = _normal(seed, 1, 2, Nq, d), _normal(seed + 1, 1, 1, Nk, d), _normal(seed + 2, 1, 1, Nk, d)
    q.zero_(), k.zero_()
    q[..., 0], q[..., 1] = 2.0 ** 10, 1
    k[..., 0] = 0 if sign > 0 else -2 * S / 2.0 ** 10
    return q, k, v


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [2, 100])
@pytest.mark.parametrize("splits", [1, 2, 3, 16])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("S,step", [(2.0 ** 21, 1), (2.0 ** 22, 0.5), (2.0 ** 23, 1), (2.0 ** 28, 32), (2.0 ** 30, 128), (2.0 ** 33, 1024)])
def test_near_scores_that_are_large(S, step, sign, splits, Nq, d):
    """Scores of S and a step or two more, in different splits, behind keys that are far below."""
    q, k, v = _one_score(S, sign, Nq, 1024, d, 20)
    for n, (key, steps) in enumerate(((40, 1), (500, 0), (700, 2), (990, 2))):
        k[0, 0, key, 0], k[0, 0, key, 1] = sign * S / 2.0 ** 10, steps * step
    _by_scores(q, k, v, 1.0, splits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [2, 100])
@pytest.mark.parametrize("splits", [1, 2, 3, 16])
def test_scores_beyond_fp32(splits, Nq, d):
    """The result of the definition, whatever the number of splits: one key has all the weight."""
    import paper_2606_07713_amd as moa
    q, k, v = _normal(30, 1, 2, Nq, d), _normal(31, 1, 1, 1000, d), _normal(32, 1, 1, 1000, d)
    q, k = (q.float() * 1e25).to(BF16), (k.float() * 1e25).to(BF16)
    for left, right in ((-1, -1), (-1, 0), (400, 0)):
        o = moa.win_attn_fwd(q, k, v, left, right, out_dtype=torch.float32, num_splits=splits)
        x = _exact(q, k, v, left, right, 0)
        s = torch.where(x.see, q.double() @ k.double().transpose(2, 3), -math.inf)
        assert torch.equal(o, v[0, 0][s.argmax(-1)].float())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [2, 100])
@pytest.mark.parametrize("splits", [1, 2, 4])
def test_scores_of_minus_infinity_count_nothing(splits, Nq, d):
    """All keys of one split or stream, or all but one of the sequence, have a score of -inf."""
    q, k, v = _normal(33, 1, 2, Nq, d), _normal(34, 1, 1, 512, d), _normal(35, 1, 1, 512, d)
    q, k = q.abs(), k.abs()
    for first, end in ((0, 64), (0, 256), (256, 512), (0, 511), (1, 512)):
        x = k.clone()
        x[:, :, first:end, 3] = -math.inf
        _check(q, x, v, num_splits=splits)


@pytest.mark.parametrize("N", [2, 40])
@pytest.mark.parametrize("splits", [1, 3, 7])
def test_scores_beyond_fp32_over_a_paged_cache(splits, N):
    """Ragged lengths, fewer new tokens than rows, a page that is not there: one key has all the weight."""
    import paper_2606_07713_amd as moa
    from test_paged_gpu import Cache, _i32
    from win_util import visible
    lens, new = [700, 90, 333], [N, 1, N - 1]
    c = Cache(lens, 2, 16, 64)
    c.table[0, 5] = -1
    c.k.copy_((c.k.float() * 1e25).to(BF16))
    q = (_normal(40, 3, 4, N, 64).float() * 1e25).to(BF16)
    for left, right, sinks in ((-1, 0, 0), (200, 0, 20)):
        out = torch.full((3, 4, N, 64), 7.0, device="cuda")
        o, lse = moa.paged_attn_fwd(q, c.k, c.v, _i32(lens), page_table=c.table, new_lens=_i32(new), left=left, right=right,
                                    sinks=sinks, out_dtype=torch.float32, num_splits=splits, out=out, return_lse=True)
        for b, n in enumerate(lens):
            (k, has), (v, _) = c.rows(c.k, b, n), c.rows(c.v, b, n)
            see = visible(torch.arange(n - new[b], n, device="cuda")[None], n, torch.tensor([n], device="cuda"), left, right, sinks) & has
            s = q[b, :, :new[b]].double() @ k.repeat_interleave(2, 0).transpose(1, 2)
            best = torch.where(see, s, -math.inf).argmax(-1)
            want = v.repeat_interleave(2, 0).gather(1, best[..., None].expand(-1, -1, 64))
            assert torch.equal(o[b, :, :new[b]].double(), want) and bool((o[b, :, new[b]:] == 7).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [2, 50])
def test_log_sums_near_zero_of_splits_by_definition(Nq, d):
    """Few keys and small scores: LSE keeps the bound of fp32 near 0, whatever the state's reference is."""
    for Nk in (1, 2, 3, 4, 7, 40):
        q, k, v = _normal(50 + Nk, 2, 16, Nq, d, std=0.1), _normal(60 + Nk, 2, 2, Nk, d, std=0.1), _normal(70 + Nk, 2, 2, Nk, d)
        v[0, 1, :1], v[1, 0, Nk - 1:] = math.nan, math.inf
        for splits in (1, 2, 3, 16):
            _check(q, k, v, num_splits=splits)
            _check(q, k, v, -1, 0, 0, num_splits=splits)
