"""Elements below the normal numbers, written into the four-bit cache."""
import pytest

from kv4_util import quantised
from test_kv4_gpu import _ints, _pool

pytestmark = pytest.mark.gpu


def test_subnormal_elements():
    # fp32 elements below the normal numbers whose nearest value is not zero: a quarter of the
    # smallest step, 2^-127, is the last that goes to zero
    import torch
    import paper_2606_07713_amd as moa
    cache, table = _pool(1, 64, 64, 1, 64, torch.Generator().manual_seed(1))
    x = torch.zeros((1, 1, 4, 64), dtype=torch.float64)
    x[0, 0, 0] = torch.linspace(0.25, 2, 64) * 2.0 ** -126
    x[0, 0, 1] = -torch.linspace(2, 0.25, 64) * 2.0 ** -127
    x[0, 0, 2, :3] = torch.tensor([1.0 + 2.0 ** -22, 1.0, 1.0 - 2.0 ** -22]) * 2.0 ** -127
    x[0, 0, 3, 40:44] = torch.tensor([1.0, -1.5, 1.75, -2.0]) * 2.0 ** -127
    k = x.float()
    assert torch.equal(k.double()[0, 0, 2], x[0, 0, 2]) and (k[0, 0, 2, :3] != 0).all()
    k = k.to("cuda")
    moa.kv4_write(k, k.flip(3), cache, _ints([4]), page_table=table)
    ko, vo = moa.kv4_read(cache, 4, 64, _ints([4]), page_table=table, out_dtype=torch.float32)
    want = quantised(k.cpu())
    assert (want[0, 0, 2, :3] != 0).tolist() == [True, False, False]
    assert torch.equal(ko.cpu().double(), want) and torch.equal(vo.cpu().double(), quantised(k.cpu().flip(3)))
