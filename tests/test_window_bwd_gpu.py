"""Gradients of the attention in a window (``win_attn_bwd``) against their definition in fp64 and
against differences of the forward."""
import math

import pytest
import torch

from test_window_gpu import WINDOWS, _exact, _normal
from win_util import close

pytestmark = pytest.mark.gpu


def _check(q, k, v, do, left=-1, right=-1, sinks=0, scale=None, o_dtype=torch.bfloat16, **given):
    import paper_2606_07713_amd as moa
    x = _exact(q, k, v, left, right, sinks, scale, do)
    o, lse = moa.win_attn_fwd(q, k, v, left, right, sinks, scale=scale, out_dtype=o_dtype, return_lse=True)
    got = moa.win_attn_bwd(q, k, v, o, do, lse, left, right, sinks, scale=scale, **given)
    torch.cuda.synchronize()
    for name, g, (want, bound) in zip("qkv", got, x.grad_bounds(o_dtype, k.shape[1])):
        assert g.dtype is torch.bfloat16
        try:
            close(g, want, bound)
        except AssertionError as e:
            raise AssertionError(f"d{name}: {e}") from None
    return got


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,Nk,G", [(1, 1, 1), (1, 300, 4), (3, 2, 2), (64, 64, 1), (200, 200, 1), (130, 333, 3), (65, 40, 2),
                                     (129, 129, 5), (400, 400, 2)])
def test_sizes(window, d, Nq, Nk, G):
    Hk = 2
    q, k, v = _normal(1, 2, Hk * G, Nq, d), _normal(2, 2, Hk, Nk, d), _normal(3, 2, Hk, Nk, d)
    _check(q, k, v, _normal(4, 2, Hk * G, Nq, d), *window)


@pytest.mark.parametrize("sinks", [1, 40, 128, 300])
@pytest.mark.parametrize("left,right", [(20, 0), (64, 30), (0, -1)])
@pytest.mark.parametrize("d", [64, 128])
def test_far_queries_of_the_first_keys(sinks, left, right, d):
    q, k, v = _normal(5, 1, 4, 1500, d), _normal(6, 1, 2, 1500, d), _normal(7, 1, 2, 1500, d)
    _check(q, k, v, _normal(8, 1, 4, 1500, d), left, right, sinks)
    q, k, v = q[:, :, :900], k[:, :, :700], v[:, :, :700]
    _check(q, k, v, _normal(9, 1, 4, 900, d), left, right, sinks)


@pytest.mark.parametrize("d", [64, 128])
def test_strided_views_and_fp32_outputs(d):
    """Slices of a packed projection output, gradients into one of the same layout."""
    B, Hq, Hk, N = 2, 6, 2, 150
    x, g = _normal(10, B, N, Hq + 2 * Hk, d).transpose(1, 2), _normal(11, B, N, Hq, d).transpose(1, 2)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    dq, dk, dv = (torch.full((B, N, h, 2 * d), 7.0, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hk, Hk))
    views = [t[..., :d].transpose(1, 2) for t in (dq, dk, dv)]
    a = _check(q, k, v, g, 40, 0, 2, dq=views[0], dk=views[1], dv=views[2])
    b = _check(*(t.contiguous() for t in (q, k, v, g)), 40, 0, 2)
    for x, y, whole in zip(a, b, (dq, dk, dv)):
        assert torch.equal(x, y) and bool((whole[..., d:] == 7).all())
    _check(q, k, v, g, 40, 0, 2, o_dtype=torch.float32)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_scales(scale):
    q, k, v = _normal(12, 1, 4, 100, 64), _normal(13, 1, 2, 120, 64), _normal(14, 1, 2, 120, 64)
    _check(q, k, v, _normal(15, 1, 4, 100, 64), 50, 0, 1, scale=scale)


def test_shared_heads_are_the_sum_of_their_copies():
    """The gradient of a shared head equals the sum of those of its copies.  The two calls round apart
    from each other -- a row's weights are taken against a reference that the other rows of its wave have
    a part in, so O, and D with it, differ in their last bits -- and each is within its own bound of the
    same exact gradient: by the triangle inequality they are within the sum of the bounds of each other."""
    q, k, v, do = _normal(16, 1, 6, 300, 64), _normal(17, 1, 2, 300, 64), _normal(18, 1, 2, 300, 64), _normal(19, 1, 6, 300, 64)
    _, dk, dv = _check(q, k, v, do, 64, 0, 3)
    kk, vv = k.repeat_interleave(3, 1), v.repeat_interleave(3, 1)
    _, ek, ev = _check(q, kk, vv, do, 64, 0, 3)
    shared = _exact(q, k, v, 64, 0, 3, do=do).grad_bounds(torch.bfloat16, 2)
    copies = _exact(q, kk, vv, 64, 0, 3, do=do).grad_bounds(torch.bfloat16, 6)
    for i, (a, b) in enumerate(((dk, ek), (dv, ev)), 1):
        off = (a.double() - b.double().view(1, 2, 3, 300, 64).sum(2)).abs()
        assert bool((off <= shared[i][1] + copies[i][1].view(1, 2, 3, 300, 64).sum(2)).all())


@pytest.mark.parametrize("d", [64, 128])
def test_differences(d):
    """Gradients of sum(do * o) against central differences of the fp32 output along random directions."""
    import paper_2606_07713_amd as moa
    t = [_normal(20 + i, 1, h, 96, d) for i, h in enumerate((4, 2, 2))]
    do = _normal(24, 1, 4, 96, d)
    how = (30, 0, 2)
    o, lse = moa.win_attn_fwd(*t, *how, out_dtype=torch.float32, return_lse=True)
    grads = moa.win_attn_bwd(*t, o, do, lse, *how)
    for i, g in enumerate(grads):
        # steps of whole bf16 units, so that both points are inputs exactly: 2^-5 up and down on a grid of 2^-6
        way = torch.randint(0, 2, t[i].shape, generator=torch.Generator().manual_seed(i)).cuda() * 2.0 - 1
        at = [x.float() for x in t]
        at[i] = (at[i] * 16).round() / 16
        point = [x.to(torch.bfloat16) for x in at]
        o, lse = moa.win_attn_fwd(*point, *how, out_dtype=torch.float32, return_lse=True)
        g = moa.win_attn_bwd(*point, o, do, lse, *how)[i]
        ends = []
        for sign in (1, -1):
            moved = list(point)
            moved[i] = (at[i] + sign * way / 64).to(torch.bfloat16)
            way_got = (moved[i].float() - point[i].float()) * sign
            ends.append((moa.win_attn_fwd(*moved, *how, out_dtype=torch.float32).double() * do.double()).sum())
        slope = (ends[0] - ends[1]) / 2
        want = (g.double() * way.double() / 64).sum()
        # Elements of 2 and more do not take the whole step.  The gradient's roundings: at most three halves of
        # bf16 steps an element, 1.2e-2 of it (P, dS, dK), of random signs under a random direction, so 1.2e-2 of
        # the norm; the third derivative, with scores that move by 2^-6 |q| and less: (2^-6 sqrt(d) / sqrt(d))^2
        # of the slope, 2.5e-4.  Four times the two.
        off = (g.double().abs() * (way.double() / 64 - way_got.double()).abs()).sum()
        noise = (g.double().square().sum().sqrt() / 64) * 0.05
        assert abs(float(slope - want)) <= float(off + noise) + 1e-4


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_what_does_not_see_each_other_has_no_part(d, what):
    """A padded end: keys, values and queries' gradients behind the real tokens hold NaN, and no real
    token's gradient knows."""
    import paper_2606_07713_amd as moa
    N, real = 200, 150
    q, k, v, do = (_normal(30 + i, 2, h, N, d) for i, h in enumerate((4, 2, 2, 4)))
    for t in (q, k, v, do):
        t[:, :, real:] = what
    for how in ((-1, 0, 0), (40, 0, 3)):
        o, lse = moa.win_attn_fwd(q, k, v, *how, return_lse=True)
        got = moa.win_attn_bwd(q, k, v, o, do, lse, *how)
        head = [t[:, :, :real].contiguous() for t in (q, k, v, do)]
        x = _exact(*head[:3], *how, do=head[3])
        bounds = x.grad_bounds(torch.bfloat16, 2)
        close(got[0][:, :, :real], *bounds[0])
        # padded queries see the real keys: what these get from them is no number, unless no real key is seen
        far = real - 41
        if how[0] >= 0:
            for g, (want, bound) in zip(got[1:], bounds[1:]):
                close(g[:, :, 3:far], want[:, :, 3:far], bound[:, :, 3:far])


@pytest.mark.parametrize("Nq,Nk,left,right,sinks", [(300, 9000, -1, -1, 0), (1500, 8300, 700, 0, 5), (4300, 8400, -1, 0, 0),
                                                     (2000, 1000, -1, 300, 0), (1000, 3000, 100, 900, 300), (3000, 2900, 2000, 0, 130)])
def test_tiles_of_different_length(Nq, Nk, left, right, sinks):
    """Few key tiles, or many of a single head, seen by many queries or by few: their parts are as long as
    each other, so tiles have different numbers of them."""
    import paper_2606_07713_amd as moa
    assert moa.moa_win_attn_bwd_workspace_bytes(1, 2, 1, Nq, Nk, 64, left, right, sinks) > 4 * 2 * Nq + (1 << 16)   # some
    q, k, v = _normal(60, 1, 2, Nq, 64), _normal(61, 1, 1, Nk, 64), _normal(62, 1, 1, Nk, 64)
    _check(q, k, v, _normal(63, 1, 2, Nq, 64), left, right, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hk,N,left,right,sinks", [(2, 2, 300, 0, 0, 0), (8, 2, 333, 1, 0, 0), (4, 4, 700, 7, 0, 1), (6, 2, 200, 5, 20, 2),
                                                      (64, 4, 600, 40, 0, 3), (4, 1, 60, -1, 0, 0)])
def test_few_keys(Hq, Hk, N, left, right, sinks, d):
    """Where a row sees a handful of keys, dP - D is a difference of near numbers: with a row's only key it
    is 0.  O as a bf16 number would leave 2^-8 of |dO| |O| there; the sum over the keys leaves fp32's."""
    import paper_2606_07713_amd as moa
    q, k, v, do = (_normal(40 + i, 2, h, N, d) for i, h in enumerate((Hq, Hk, Hk, Hq)))
    x = _exact(q, k, v, left, right, sinks, None, do)
    o, lse = moa.win_attn_fwd(q, k, v, left, right, sinks, return_lse=True)
    got = moa.win_attn_bwd(q, k, v, o, do, lse, left, right, sinks)
    for name, g, (want, bound) in zip("qkv", got, x.grad_bounds(torch.bfloat16, Hk, few_keys=True)):
        try:
            close(g, want, bound)
        except AssertionError as e:
            raise AssertionError(f"d{name}: {e}") from None


def test_nothing_to_do():
    import paper_2606_07713_amd as moa
    for B, Hq, Nq, Nk in ((0, 2, 3, 4), (1, 0, 3, 4), (1, 2, 0, 4), (2, 2, 3, 0)):
        q, k = _normal(1, B, Hq, Nq, 64), _normal(2, B, 1, Nk, 64)
        o, lse = moa.win_attn_fwd(q, k, k, 3, 0, return_lse=True)
        dq, dk, dv = moa.win_attn_bwd(q, k, k, o, q, lse, 3, 0)
        assert all(bool((t == 0).all()) for t in (dq, dk, dv))


def test_a_training_step_in_a_graph():
    """Forward and gradients captured once, replayed on new inputs, with eager work between: the same bits."""
    import paper_2606_07713_amd as moa
    t = [_normal(40 + i, 1, h, 700, 64) for i, h in enumerate((8, 2, 2, 8))]
    how = (99, 0, 4)

    def step(q, k, v, do):
        o, lse = moa.win_attn_fwd(q, k, v, *how, return_lse=True)
        return o, *moa.win_attn_bwd(q, k, v, o, do, lse, *how)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*t)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*t)
    for i in range(3):
        new = [_normal(50 + 4 * i + j, *x.shape) for j, x in enumerate(t)]
        for x, y in zip(t, new):
            x.copy_(y)
        graph.replay()
        want = step(*new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
