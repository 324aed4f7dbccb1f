"""The attention over the four-bit cache against fp64 over the stored values: bounds of a few units of
fp32 but for the weights' own 2^-18 and the output's rounding (``kv4_util.attention_error``), and
nothing that is NaN or infinite where the definition is not."""
import pytest

import test_kv4_gpu
from kv4_util import attention, attention_error, stored
from test_kv4_gpu import ATTNS, _cache_of, _ints, _pool

pytestmark = pytest.mark.gpu


def check(q, cache, table, page, lens, new, causal, scale, o, lse):
    """O and LSE of every head against fp64."""
    import torch
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[o.dtype]
    B, Hq, N, d = q.shape
    G = Hq // cache.shape[1]
    host, tab = cache.cpu(), None if table is None else table.cpu()
    scale = float(torch.tensor(d ** -0.5).float()) if scale is None else scale
    worst = [0.0, 0.0]
    for b in range(B):
        K, V = stored(host, page, d, tab, b, lens[b])
        n = N if new is None else new[b]
        seen = torch.arange(n) + lens[b] - n + 1 if causal else torch.full((n,), lens[b])
        for h in range(Hq):
            ref = attention(q[b, h, :n].cpu().double(), K[h // G], V[h // G], seen, scale)
            got = attention_error(o[b, h, :n].cpu().double(), lse[b, h, :n].cpu().double(), ref, lens[b], d, half)
            assert not isinstance(got, str), (b, h, got)
            worst = [max(x, y) for x, y in zip(worst, got)]
    print(f"  O worst {worst[0]:.2f} of the bound, LSE {worst[1]:.2f}", flush=True)
    assert worst[0] <= 1 and worst[1] <= 1


@pytest.mark.parametrize("case", ATTNS, ids=lambda c: "x".join(map(str, c[:6])) + f"_{max(c[6])}_{'c' if c[8] else 'f'}")
def test_weights_keep_their_digits(case):
    import torch
    import paper_2606_07713_amd as moa
    B, Hq, Hk, N, d, page, lens, new, causal, scale, splits, _ = case
    print(f"kv4 attention, fp32 out {case}", flush=True)
    cache, table = _cache_of(B, Hk, d, page, lens)
    q = torch.randn((B, N, Hq, d), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to("cuda").transpose(1, 2)
    o, lse = moa.kv4_attn_fwd(q, cache, _ints(lens), page_table=table, new_lens=None if new is None else _ints(new),
                              causal=causal, scale=scale, num_splits=splits, out_dtype=torch.float32, return_lse=True)
    torch.cuda.synchronize()
    check(q, cache, table, page, lens, new, causal, scale, o, lse)


@pytest.mark.parametrize("d,N,splits", [(64, 1, 1), (128, 1, 3), (128, 40, 1)])
def test_values_near_the_largest_that_the_format_holds(d, N, splits):
    # later keys weigh up to 2^14 times the first tile's, the values are +-2^112 to 6 * 2^112: sums of 2^14 V
    # leave fp32, the results do not
    import torch
    import paper_2606_07713_amd as moa
    n, page = 64 * 24, 64
    cache, table = _pool(1, n, page, 1, d, torch.Generator().manual_seed(1))
    gen = torch.Generator().manual_seed(2)
    k = torch.zeros((1, 1, n, d))
    k[0, 0, :, 0] = torch.arange(n) // 64 // 12 * 8.0 + torch.randint(0, 3, (n,), generator=gen)
    v = torch.randint(1, 7, (1, 1, n, d), generator=gen) * 2.0 ** 112
    v[0, 0, :, ::2] *= -1
    moa.kv4_write(k.to("cuda"), v.to("cuda"), cache, _ints([n]), page_table=table)
    q = torch.zeros((1, 1, N, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    o, lse = moa.kv4_attn_fwd(q, cache, _ints([n]), page_table=table, scale=1.0, num_splits=splits, return_lse=True,
                              out_dtype=torch.float32)
    torch.cuda.synchronize()
    check(q, cache, table, page, [n], None, False, 1.0, o, lse)


def test_scores_that_leave_fp32_do_not_pass_for_rows_that_see_nothing():
    # scores of +-2^126 times 8: the row is NaN; a score that overflows downwards beside others weighs nothing
    import torch
    import paper_2606_07713_amd as moa
    cache, table = _pool(1, 1024, 64, 1, 64, torch.Generator().manual_seed(1))
    for n, splits in ((3, 1), (700, 1), (700, 4)):
        k = torch.zeros((1, 1, n, 64), device="cuda")
        v = torch.ones_like(k)
        for sign in (1.0, -1.0):
            k[..., 0] = sign * 2.0 ** 63
            moa.kv4_write(k, v, cache, _ints([n]), page_table=table)
            q = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
            q[..., 0] = 2.0 ** 63
            o, lse = moa.kv4_attn_fwd(q, cache, _ints([n]), page_table=table, scale=8.0, num_splits=splits, return_lse=True)
            assert torch.isnan(o).all(), (n, splits, sign)
            assert torch.equal(lse, torch.full_like(lse, sign * float("inf"))), (n, splits, sign)
        k[..., ::3, 0] = 0
        moa.kv4_write(k, v, cache, _ints([n]), page_table=table)
        o, lse = moa.kv4_attn_fwd(q, cache, _ints([n]), page_table=table, scale=8.0, num_splits=splits, return_lse=True,
                                  out_dtype=torch.float32)
        want = torch.tensor(float(-(-n // 3)), dtype=torch.float64).log()
        # equal weights of one: sums exact, a logarithm and its products
        assert (o == 1).all() and ((lse.cpu().double() - want).abs() <= 4 * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("test,args", [
    ("test_no_page_table_and_strided_output", ()),
    *[("test_nan_blocks_reach_only_the_rows_that_see_them", (n, causal, d))
      for n, causal in ((1, True), (7, True), (40, True), (5, False)) for d in (64, 128)],
    ("test_extreme_scores", ()),
    ("test_norm_rope_write_attend_together", ()),
    ("test_pool_beyond_four_gigabytes", ()),
], ids=lambda v: v if isinstance(v, str) else "_".join(map(str, v)))
def test_no_log_sum_is_nan_where_a_row_sees_a_key(monkeypatch, test, args):
    # the calls of test_kv4_gpu whose own check takes a NaN log sum for 0
    monkeypatch.setattr(test_kv4_gpu, "_check_attn", check)
    getattr(test_kv4_gpu, test)(*args)
