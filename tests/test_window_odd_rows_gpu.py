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
