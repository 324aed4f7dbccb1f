"""Appending to the paged bf16 cache with positions on several axes (``paged_append`` with ``sections``),
against the rotation's definition in fp64 and the bits of ``qk_norm_rope``."""
import pytest
import torch

from test_paged_gpu import Cache, _freq, _i32, _normal
from win_util import EPS, close

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _turned(x, w, pos, freq, sections, interleaved):
    """x [B, H, N, d] normed and turned in fp64, the pairs of section a by positions pos[a] [B, N]; and the
    size of each result's terms."""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
    r = 2 * freq.shape[0]
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections)).cuda()
    at = pos.double()[axis].movedim(0, -1) * freq.double()           # [B, N, r / 2]
    cos, sin = at.cos()[:, None], at.sin()[:, None]
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    out, size = x.clone(), x.abs()
    out[..., i], out[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., j] * cos + x[..., i] * sin
    size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return out, size


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot,sections", [(64, 64, (8, 12, 12)), (128, 128, (16, 24, 24)), (128, 96, (0, 40, 1, 7)), (64, 32, (16,)),
                                            (128, 64, (31, 1))])
@pytest.mark.parametrize("N,norm", [(1, False), (37, True)])
def test_sections(N, norm, d, rot, sections, interleaved, dtype):
    import paper_2606_07713_amd as moa
    B, Hq, Hk = 3, 6, 2
    c = Cache([N, 90 + N, 40 + N], Hk, 16, d)
    q, k, v = (_normal(s, B, h, N, d, std=2.0, dtype=dtype) for s, h in ((1, Hq), (2, Hk), (3, Hk)))
    wq, wk = (_normal(s, d, dtype=dtype) + 1 for s in (4, 5)) if norm else (None, None)
    freq, g = _freq(rot), torch.Generator().manual_seed(6)
    pos = torch.randint(-50, 5000, (len(sections), B, N), generator=g).cuda()
    got = moa.paged_append(q, k, v, c.k, c.v, _i32(c.lens), page_table=c.table, positions=pos, inv_freq=freq, q_weight=wq,
                           k_weight=wk, interleaved=interleaved, sections=sections)
    torch.cuda.synchronize()
    rows = [torch.stack([c.rows(pool, b, n)[0][:, n - N:] for b, n in enumerate(c.lens)]) for pool in (c.k, c.v)]
    assert torch.equal(rows[1], v.to(BF16).double())
    for out, x, w in ((got, q, wq), (rows[0], k, wk)):
        want, size = _turned(x, w, pos, freq, sections, interleaved)
        # angle in fp32 turns (2^-23), sine and cosine, rsqrt and the mean (2^-20 together), one rounding
        close(out, want, want.abs() * EPS[BF16] + size * 2.0 ** -19 + 1e-30)
    if dtype is BF16:
        a, b = moa.qk_norm_rope(q, k, positions=pos, inv_freq=freq, q_weight=wq, k_weight=wk, interleaved=interleaved,
                                sections=sections)
        assert torch.equal(got, a) and torch.equal(rows[0], b.double())


@pytest.mark.parametrize("N", [2, 20])
def test_places_on_every_axis(N):
    """Without positions every axis has the token's place in its sequence: as with one axis."""
    import paper_2606_07713_amd as moa
    lens, new = [N + 7, 64, 100], [N, 1, N - 1]
    q, k, v = _normal(1, 3, 4, N, 64), _normal(2, 3, 2, N, 64), _normal(3, 3, 2, N, 64)
    both = []
    for sections in (None, (8, 20, 4)):
        c = Cache(lens, 2, 32, 64)
        out = torch.zeros_like(q)
        moa.paged_append(q, k, v, c.k, c.v, _i32(lens), page_table=c.table, new_lens=_i32(new), inv_freq=_freq(64),
                         sections=sections, q_out=out)
        both.append((out, c.k, c.v))
    assert all(torch.equal(a, b) for a, b in zip(*both))
