"""The checks of the attention over the four-bit cache find what they are for, on the CPU: mistakes
planted in results that are otherwise right."""
import pytest
import torch

from kv4_util import attention, attention_error


def _case(n=5, m=40, d=64):
    g = torch.Generator().manual_seed(4)
    q, K, V = (torch.randn((k, d), generator=g).double() for k in (n, m, m))
    return attention(q, K, V, torch.tensor([0, 1, 7, m, m]), 0.125), m, d


def test_right_results_pass():
    (o, lse, *rest), m, d = _case()
    got = attention_error(o.float().double(), lse.float().double(), (o, lse, *rest), m, d)
    assert not isinstance(got, str) and max(got) <= 1


@pytest.mark.parametrize("wrong", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("row", [1, 3])
def test_a_log_sum_that_is_no_number_is_found(wrong, row):
    ref, m, d = _case()
    lse = ref[1].clone()
    lse[row] = wrong
    assert attention_error(ref[0], lse, ref, m, d).startswith("LSE")


def test_empty_rows_and_small_errors_are_found():
    ref, m, d = _case()
    o, lse = ref[0].clone(), ref[1].clone()
    lse[0] = 0.0                                # a row that sees nothing has none
    assert attention_error(o, lse, ref, m, d).startswith("LSE")
    o[3, 5] += 2.0 ** -9 * ref[2][3, 5]          # a weight's rounding to one bf16 number
    assert attention_error(o, ref[1], ref, m, d)[0] > 1
    lse = ref[1].clone()
    lse[3] += 1e-4
    assert attention_error(ref[0], lse, ref, m, d)[1] > 1
    o[1, 0] = float("nan")
    assert attention_error(o, ref[1], ref, m, d).startswith("O")
