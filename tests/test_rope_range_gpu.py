"""Head norms with rotation on rows whose squares leave fp32: tiny ones (without an eps that hides
them) and huge ones, against the formulas in fp64, in the bounds of ``test_rope_gpu``."""
import pytest

from test_rope_gpu import _angles, _near, _reference

pytestmark = pytest.mark.gpu


def _rows(d, dtype, exponents, seed=1):
    """One head of random rows [1, 1, n, d], one for each exponent, of elements near 2^exponent, and
    one of very different elements: 1 among such."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((1, 1, len(exponents), d), generator=g, dtype=torch.float64).clamp(-1.9, 1.9)
    x = (x * torch.exp2(torch.tensor(exponents, dtype=torch.float64))[:, None]).to(dtype)
    return x


@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,eps,exponents", [
    ("f32", 0.0, [-60, -66, -70, -72, -73, -76, -80, -100, -120]),
    ("bf16", 0.0, [-50, -66, -72, -80, -118]),
    ("f32", 2.0 ** -140, [-66, -70, -71, -76, -100, 0]),
    ("f32", 2.0 ** -96, [-44, -48, -60, -100]),
    ("f32", 1e-6, [0, 58, 59, 60, 61, 62, 64, 100, 126]),
    ("bf16", 0.0, [0, 60, 62, 80, 126, -70]),
], ids=lambda v: str(v) if not isinstance(v, list) else "_".join(map(str, v)))
def test_rows_whose_squares_leave_fp32(dtype, eps, exponents, d, il):
    import torch
    import paper_2606_07713_amd as moa
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    print(f"rows of 2^{exponents} {dtype} eps {eps} d {d}", flush=True)
    q = _rows(d, dt, exponents)
    n = len(exponents)
    w = torch.linspace(0.5, 2.0, d)
    freq = torch.tensor([10000.0 ** (-4 * i / d) for i in range(d // 4)], dtype=torch.float32)
    pos = torch.arange(n)[None] + 5
    how = dict(positions=pos.to("cuda"), inv_freq=freq.to("cuda"), q_weight=w.to("cuda"), eps=eps, interleaved=il)
    ang = _angles(pos, freq, None, 1, n)
    # gradients of a size that leaves those of x in the type's normal numbers, as far as one size for
    # both does
    size = torch.exp2(torch.tensor([max(-40, min(40, e)) for e in exponents]).float())[:, None]
    dy = (torch.randn(q.shape, generator=torch.Generator().manual_seed(2)) * size).to(dt)
    y, _ = moa.qk_norm_rope(q.to("cuda"), **how)
    dq, _, dw, _ = moa.qk_norm_rope_bwd(q.to("cuda"), None, dy.to("cuda"), None, **how)
    torch.cuda.synchronize()
    # eps as the call takes it
    ref = _reference(q, w, ang, il, float(torch.tensor(eps, dtype=torch.float32)), dy)
    _near("y", y, *ref[:2])
    # results below 2^-126 have 2^-149 (bf16: 2^-133) for a step
    tiny = 2.0 ** (-149 if dt == torch.float32 else -133)
    _near("dq", dq, ref[2], ref[3] + tiny)
    _near("dw", dw, *ref[4:])


@pytest.mark.parametrize("d", [64, 128])
def test_an_infinite_element_makes_the_others_zero(d):
    # x / sqrt(inf): 0, and NaN in the infinity's own pair
    import torch
    import paper_2606_07713_amd as moa
    q = torch.full((1, 1, 2, d), 3e38)
    q[0, 0, 1] = 1.0
    q[0, 0, :, 5] = torch.inf
    w = torch.full((d,), 2.0, device="cuda")
    freq = torch.full((d // 2,), 0.5, device="cuda")
    y, _ = moa.qk_norm_rope(q.to("cuda"), inv_freq=freq, q_weight=w)
    bad = torch.isnan(y).cpu()
    assert bad[..., [5, 5 + d // 2]].all() and bad.sum() == 4
    assert not torch.nan_to_num(y).any()
