"""What the element-by-element tolerances of the paged attention can tell apart, shown on the CPU with emulated mistakes."""
import pytest
import torch

from paged_bounds import Exact
from paged_reference import PagedMirror

BF, HF = torch.bfloat16, torch.float16
# lens, H, D, G, type, scale: small scales keep the scores' own error below a rounding of P. Of fp16 only few rows tell: a rounding of
# P is off by 2^-11 / sqrt(12) of a row's share at most in the mean square, over 170 to 300 rows about 2^-11 / sqrt(12 * 170) = 1.1e-5 of
# the sum of p |v|, three times that at the worst element, against (2 (300 / 4 + 32) + 16 + 7) 2^-23 + 2^-19 + ... = 3.5e-5 allowed.
CASES = [([3, 40, 0, -1, 129], 2, 64, 4, BF, 0.02), ([300, 260], 3, 64, 3, BF, 0.02), ([300, 170], 2, 128, 9, HF, 0.02),
         ([17, 64], 4, 128, 1, HF, 0.02), ([300, 260], 2, 128, 16, BF, 0.01)]


def inputs(case):
    lens, H, D, G, dt, scale = case
    m = PagedMirror(lens, H, D, 16, max(lens) + 8, dt, device=None, G=G)
    g = torch.Generator().manual_seed(len(lens) + D)
    q, k, v = (torch.randn(len(lens), h, D, generator=g).to(dt) for h in (H * G, H, H))
    return m, q, k, v, scale


@pytest.mark.parametrize("case", CASES)
def test_a_single_rounding_of_p_is_outside(case):
    m, q, k, v, scale = inputs(case)
    e = Exact(m, q, k, v, scale)
    if case[4] == HF and max(case[0]) > 100:
        e.assert_out(e.out.to(m.dtype))
        return
    with pytest.raises(AssertionError):
        e.assert_out(e.with_rounded_p(m.dtype).to(m.dtype))
    with pytest.raises(AssertionError):
        e.assert_out(e.with_rounded_p(m.dtype))
    e.assert_out(e.out.to(m.dtype))


def test_rows_that_gain_nothing_are_outside():
    m = PagedMirror([20000], 1, 64, 64, 20000, device=None)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(1, h, 64, generator=g).bfloat16() for h in (4, 1, 1))
    e = Exact(m, q, k, v, 0.125, decay=0.75)
    held = e.weight_tol > 0
    assert int(held.sum()) == 20000
    assert bool((e.gain[held] > 10 * e.weight_tol[held]).all())           # also the lightest row's gain counts
    e.assert_weights(e.weight.float(), e.w_new)
    with pytest.raises(AssertionError):
        e.assert_weights((e.weight - e.gain).float(), e.w_new)


def test_the_exact_form_matches_the_row_by_row_one():
    m, q, k, v, scale = inputs(([9, 0, -1, 70], 2, 64, 3, BF, 0.125))
    e = Exact(m, q, k, v, scale, decay=0.5)
    (out, lse, w_new), _, _ = m.attention(q, k, v, scale, True, 0.5)
    assert torch.allclose(e.out.view_as(out), out) and torch.allclose(e.lse.view_as(lse), lse) and torch.allclose(e.w_new, w_new)
    assert torch.allclose(e.weight.nan_to_num(-1.0), m.weight.nan_to_num(-1.0))
