"""Which views may interleave in one buffer in moa_rope.h's calls: on the CPU, where a call that is
not refused fails for want of a device, and such a call on the GPU."""
import pytest

moa = pytest.importorskip("paper_2606_07713_amd", reason="HIP library not built")
from test_rope_kv4_api import P, _rope, _rope_bwd  # noqa: E402


@pytest.fixture
def no_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("calls that are not refused would run on the GPU")


# [N][B][8 heads][d]: heads of one token and batch entry together, batches the inner dimension
TOKENS_FIRST = [8 * 64, 64, 2 * 8 * 64]


@pytest.mark.usefixtures("no_device")
def test_packed_heads_with_the_tokens_first_take_turns():
    q, k = P, P + 4 * 64 * 2       # four heads of queries, then two of keys
    views = dict(qs=TOKENS_FIRST, ks=TOKENS_FIRST, qos=TOKENS_FIRST, kos=TOKENS_FIRST)
    assert _rope(Q=q, K=k, Qo=q, Ko=k, **views) == moa.MOA_ERR_HIP
    assert _rope(Q=2 * P, K=3 * P, Qo=q, Ko=k, qos=TOKENS_FIRST, kos=TOKENS_FIRST) == moa.MOA_ERR_HIP
    grads = dict(dqos=TOKENS_FIRST, dkos=TOKENS_FIRST, dqs=TOKENS_FIRST, dks=TOKENS_FIRST)
    k = P + 4 * 64 * 4             # fp32 there
    assert _rope_bwd(Q=13 * P, K=14 * P, dQo=P, dKo=k, dQ=P, dK=k, **grads) == moa.MOA_ERR_HIP


@pytest.mark.usefixtures("no_device")
def test_packed_heads_that_meet_stay_refused():
    q = P
    for k in (P + 3 * 64 * 2, P + 4 * 64 * 2 - 16, P + 7 * 64 * 2):    # keys begin in the queries, or end in the next entry's
        assert _rope(Q=2 * P, K=3 * P, Qo=q, Ko=k, qos=TOKENS_FIRST, kos=TOKENS_FIRST) == moa.MOA_ERR_INVALID_ARG
    # other strides than each other's: not told apart
    other = [8 * 64, 64, 3 * 8 * 64]
    assert _rope(Q=2 * P, K=3 * P, Qo=q, Ko=P + 4 * 64 * 2, qos=TOKENS_FIRST, kos=other) == moa.MOA_ERR_INVALID_ARG
    # tokens closer together than the batches of one
    near = [8 * 64, 64, 8 * 64 + 512]
    assert _rope(Q=2 * P, K=3 * P, Qo=q, Ko=P + 4 * 64 * 2, B=4, qos=near, kos=near) == moa.MOA_ERR_INVALID_ARG


@pytest.mark.gpu
def test_in_place_with_the_tokens_first():
    import torch
    g = torch.Generator().manual_seed(1)
    x = torch.randn((37, 3, 8, 64), generator=g).to(torch.bfloat16).to("cuda")     # [N][B][heads][d]
    q, k = x[:, :, :4].permute(1, 2, 0, 3), x[:, :, 4:6].permute(1, 2, 0, 3)
    w = torch.linspace(0.5, 1.5, 64, device="cuda")
    how = dict(inv_freq=torch.linspace(1.0, 0.01, 32, device="cuda"), q_weight=w, k_weight=w)
    want = moa.qk_norm_rope(q.contiguous(), k.contiguous(), **how)
    rest = x[:, :, 6:].clone()
    moa.qk_norm_rope(q, k, q_out=q, k_out=k, **how)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, :, 6:], rest)
