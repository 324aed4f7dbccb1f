"""The attention over the four-bit cache, with fp32 outputs, against fp64 over the stored values:
bounds of a few units of fp32 but for the weights' own 2^-18 (``kv4_util.attention_error``)."""
import pytest

from kv4_util import attention, attention_error, stored
from test_kv4_gpu import ATTNS, _cache_of, _ints

pytestmark = pytest.mark.gpu


def check(q, cache, table, page, lens, new, causal, scale, o, lse):
    """O and LSE (fp32) of every head against fp64."""
    import torch
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
            got = attention_error(o[b, h, :n].cpu().double(), lse[b, h, :n].cpu().double(), ref, lens[b], d)
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
