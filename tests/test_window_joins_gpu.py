"""Attention in a window: states of key streams and key splits whose references lie far apart, against
the definition in fp64.

With many rows a state's reference is the largest score of the first 32 keys that a row sees in it, and
its sums may be up to 2^127 against that: the state with the lower reference can hold most of a row."""
import math

import pytest
import torch

from test_window_bwd_gpu import _check as check_gradients
from test_window_gpu import _exact, _normal
from win_util import close

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def close_lse(got, want, bound):
    """LSE as it is: NaN where it is no number, -inf where nothing is visible, else within the bound."""
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got == -math.inf, want == -math.inf)
    real = want.isfinite()
    close(torch.where(real, got.double(), 0.0), torch.where(real, want, 0.0), torch.where(real, bound, 1.0))


def _check(q, k, v, left=-1, right=-1, sinks=0, scale=None, num_splits=0):
    import paper_2606_07713_amd as moa
    x = _exact(q, k, v, left, right, sinks, scale)
    many = q.shape[2] * (q.shape[1] // k.shape[1]) > 32
    for dt in (BF16, torch.float32):
        o, lse = moa.win_attn_fwd(q, k, v, left, right, sinks, scale=scale, out_dtype=dt, return_lse=True, num_splits=num_splits)
        torch.cuda.synchronize()
        close(o, x.o, x.o_bound(dt, 3 if dt is torch.float32 else 1 if many else 2), x.odd)
        close_lse(lse, x.lse, x.lse_bound())


def _inputs(Nq, G, Nk, d, at, base=0.0, B=1, Hk=1, seed=1):
    """Scores in log2 units (with scale = ln 2): `base`, or what `at` has for keys from the first to behind
    the last.  Values of 2^-6, so that sums of weights up to 2^119.5 and 256 of them stay in fp32."""
    q, k, v = _normal(seed, B, Hk * G, Nq, d), _normal(seed + 1, B, Hk, Nk, d), _normal(seed + 2, B, Hk, Nk, d, std=2.0 ** -6)
    q.zero_()
    q[..., 0] = 1
    k[..., 0] = base
    for first, end, score in at:
        k[:, :, first:end, 0] = score
        assert float(k[0, 0, first, 0]) == score     # a bf16 number
    return q, k, v


# Key 40 lies behind the first 32 of tile 0, the peak in the first 32 keys of another stream's or split's
# first tile: (splits, its key of 1024).
PEAKS = [(1, 64), (2, 512), (3, 384), (16, 64), (16, 960)]
LEVELS = [(100, 127), (119, 125.5), (119.5, 127), (119.5, 130), (126, 127), (126.5, 126.5), (126.5, 127), (126.5, 140), (127, 150),
          (110, 252), (140, 126), (140, 150)]   # rise of key 40, peak


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,G", [(1, 2), (20, 1), (90, 2)])
@pytest.mark.parametrize("splits,key", PEAKS)
def test_references_far_apart(splits, key, Nq, G, d):
    for rise, peak in LEVELS:
        q, k, v = _inputs(Nq, G, 1024, d, [(40, 41, rise), (key, key + 1, peak)])
        for window in ((-1, -1, 0), (-1, 0, 0), (300, 0, 100)):
            _check(q, k, v, *window, scale=math.log(2), num_splits=splits)


@pytest.mark.parametrize("Nq,G", [(4, 2), (90, 2)])
@pytest.mark.parametrize("splits", [2, 16])
def test_a_split_by_definition_beside_others(splits, Nq, G):
    """Split 0 holds 2^119 against its reference of 0, the last one starts at -30 and rises by 130, which
    leaves fp32: it is done by the definition, whose state has a reference of its own."""
    for low, top in ((119, 100), (100, 100), (90, 119), (119.5, 119)):
        q, k, v = _inputs(Nq, G, 1024, 64, [(960, 992, -30.0), (1000, 1001, top), (40, 41, low)])
        _check(q, k, v, scale=math.log(2), num_splits=splits)


def test_many_small_splits_beside_a_high_one():
    """Every split but one holds 2^119.5: together a tenth of the row, each by itself 2^-7.5 of it."""
    q, k, v = _inputs(90, 2, 1024, 64, [*((40 + 64 * s, 41 + 64 * s, 119.5) for s in range(15)), (960, 961, 127)])
    v[..., 0] = 2.0 ** -5
    _check(q, k, v, scale=math.log(2), num_splits=16)


def test_splits_of_many_workgroups():
    """More workgroups than compute units: one key stream each."""
    for rise, peak in ((119.5, 127), (110, 130), (119.5, 126.5)):
        q, k, v = _inputs(64, 1, 512, 128, [(40, 41, rise), (256, 257, peak)], B=20, Hk=8)
        _check(q, k, v, scale=math.log(2), num_splits=2)


@pytest.mark.parametrize("d", [64, 128])
def test_wide_scores(d):
    """Scores with a deviation of 45 and more: references and peaks of all states differ."""
    for std in (3, 7, 12):
        q, k, v = _normal(5, 1, 4, 90, d, std=std), _normal(6, 1, 2, 1000, d, std=std), _normal(7, 1, 2, 1000, d)
        for splits in (1, 2, 8):
            _check(q, k, v, -1, 0, 0, num_splits=splits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Nk", [(90, 128), (90, 1024), (300, 300)])
def test_gradients_of_references_far_apart(Nq, Nk, d):
    do = _normal(9, 1, 2, Nq, d)
    for rise, peak in ((126.5, 127), (126, 127), (119.5, 127), (110, 130), (140, 150)):
        q, k, v = _inputs(Nq, 2, Nk, d, [(40, 41, rise), (64, 65, peak)])
        check_gradients(q, k, v, do, scale=math.log(2))


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_wide_scores(d):
    for std in (3, 7):
        q, k, v = _normal(15, 1, 4, 200, d, std=std), _normal(16, 1, 2, 500, d, std=std), _normal(17, 1, 2, 500, d)
        check_gradients(q, k, v, _normal(18, 1, 4, 200, d), -1, 0, 0)
