"""Limits of moa_kv4.h that the host checks, on the CPU (no call here has a device to run on)."""
import pytest

moa = pytest.importorskip("paper_2606_07713_amd", reason="HIP library not built")
from test_rope_kv4_api import _attn, _rows  # noqa: E402


@pytest.mark.parametrize("scale", [3e38, -3e38, 2.0 ** 127 * 1.0001])
def test_scales_whose_product_with_log2_e_leaves_fp32_are_refused(scale):
    assert _attn(scale=scale) == moa.MOA_ERR_UNSUPPORTED
    assert _attn(scale=scale, B=0) == moa.MOA_ERR_UNSUPPORTED
    assert _attn(scale=2.0 ** 127, B=0) == _attn(scale=-(2.0 ** 127), B=0) == moa.MOA_OK


# rows may overlap, so few bytes make a call of as many tokens as there are
@pytest.mark.parametrize("name", ["moa_kv4_write"])
@pytest.mark.parametrize("d,B,Hk,N,status", [
    (128, 1, 1, (1 << 30) - 7, 2),             # (N + 6) / 4 groups of 16 lanes: 2^24 workgroups, 2^32 threads
    (128, 1, 1, (1 << 30) - 70, 4),            # a workgroup less: taken, and there is no device here
    (128, 2, 2, (1 << 28) - 7, 2),             # 4 (2^26 - 1) groups: 2^24 workgroups
    (128, 4, 64, (1 << 22) - 7, 4),            # 256 (2^20 - 1) groups: 2^24 - 16
    (64, 1, 1, (1 << 30) - 7, 4),              # 32 groups a workgroup: the sizes' own limit comes first
])
def test_rows_beyond_one_launch_are_refused(name, d, B, Hk, N, status):
    import torch
    if torch.cuda.is_available() and status == 4:
        pytest.skip("would run on the GPU")
    assert _rows(getattr(moa, name), d=d, B=B, Hk=Hk, N=N, ks=[0, 0, 0], vs=[0, 0, 0], c=1 << 40) == status


def test_read_rows_beyond_one_launch_are_refused():
    N = (1 << 30) - 7       # 2^37 elements of each, side by side
    a, b = 1 << 44, 1 << 45
    assert _rows(moa.moa_kv4_read, d=128, B=1, Hk=1, N=N, a=a, b=b) == 2
