"""Limits of moa_kv4.h that the host checks, on the CPU (no call here has a device to run on)."""
import pytest

moa = pytest.importorskip("paper_2606_07713_amd", reason="HIP library not built")
from test_rope_kv4_api import _attn  # noqa: E402


@pytest.mark.parametrize("scale", [3e38, -3e38, 2.0 ** 127 * 1.0001])
def test_scales_whose_product_with_log2_e_leaves_fp32_are_refused(scale):
    assert _attn(scale=scale) == moa.MOA_ERR_UNSUPPORTED
    assert _attn(scale=scale, B=0) == moa.MOA_ERR_UNSUPPORTED
    assert _attn(scale=2.0 ** 127, B=0) == _attn(scale=-(2.0 ** 127), B=0) == moa.MOA_OK
