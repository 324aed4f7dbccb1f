"""Limits of moa_window.h and moa_paged.h on the CPU: calls beyond them are refused before any launch (no
compute calls here)."""
import pytest

moa = pytest.importorskip("paper_2606_07713_amd", reason="HIP library not built")

P = 1 << 40          # addresses that nothing is read at: every call here is refused


def _fwd(Nq, splits, ws=None, wsn=0, B=1, H=1):
    return moa.moa_win_attn_fwd(P, 2 * P, 3 * P, 4 * P, None, B, H, H, Nq, 8, 64, None, None, None, None, -1, 0, 0, 1.0,
                                moa.MOA_BF16, ws, wsn, splits, None)


def _paged(N, splits, ws=None, wsn=0):
    return moa.moa_paged_attn_fwd(P, 2 * P, 3 * P, 4 * P, None, 5 * P, None, 6 * P, 1, 1, 1, N, 64, 16, 20, 4, 0, None, None, None,
                                  None, -1, 0, 0, 1.0, moa.MOA_BF16, ws, wsn, splits, None)


@pytest.mark.parametrize("call", [_fwd, _paged])
def test_rows_that_one_join_takes(call):
    """Four rows a workgroup of 256 threads, which one launch counts in 32 bits: 2^26 - 4 rows."""
    for splits in (2, 3, 8):
        for rows in ((1 << 26) - 3, (1 << 26) - 1):
            assert call(rows, splits, 7 * P, 1 << 39) == 2
        assert call((1 << 26) - 4, splits) == 3          # only the workspace is missing
    assert call(1 << 26, 1) == 2 and call(1 << 26, 2, 7 * P, 1 << 39) == 2


def test_choices_for_as_many_rows():
    """Calls that are refused need no workspace; the library's own choice is not to split them."""
    most = (1 << 26) - 1
    for rows, H in ((most, 1), (most // 3, 3), (1 << 25, 1)):
        assert moa.moa_win_attn_num_splits(1, H, H, rows, 8, 64, -1, 0, 0, 0) == 1
        assert moa.moa_win_attn_workspace_bytes(1, H, H, rows, 8, 64, -1, 0, 0, 0) == 0
    assert moa.moa_win_attn_workspace_bytes(1, 1, 1, most, 8, 64, -1, 0, 0, 2) == 0
    assert moa.moa_win_attn_workspace_bytes(1, 1, 1, most - 3, 8, 64, -1, 0, 0, 2) > 0
