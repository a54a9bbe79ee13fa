"""Attention over a paged cache at scores that fp32 holds in steps of more than one."""
import math

import pytest
import torch

from paged_reference import PagedMirror
from test_paged_gpu import BF, HF
from test_paged_precision_gpu import call

pytestmark = pytest.mark.gpu


def steep_scores(dt, factors, a, D=64):
    """One problem whose rows score a * factor * D exactly, by vectors of equal entries."""
    L = len(factors)
    m = PagedMirror([L], 1, D, 16, L + 8, dt)
    page, slot = m.where(0, L)
    K = torch.tensor(factors)[:, None, None].expand(L, 1, D)
    assert torch.equal(K.to(dt).float(), K)
    m.K[page, :, slot] = K.to(dt)
    m.dev["K"].copy_(m.K)
    return m, torch.full((1, 2, D), a).to(dt)


@pytest.mark.parametrize("dt,a,scale", [(BF, 2.0 ** 20, 0.1), (BF, 2.0 ** 24, 0.3), (BF, -(2.0 ** 28), 0.0884), (HF, 32768.0, 0.1), (HF, -65504.0, 0.75),
                                        (BF, 2.0 ** 20, 3.0e-3), (HF, 1024.0, 1.0)])
@pytest.mark.parametrize("L", [3, 40, 700])
def test_scores_far_beyond_what_a_rounding_of_the_maximum_allows(dt, a, scale, L):
    """Scores of 2^25 to 2^42, where one step of fp32 is more than the softmax can tell apart: only the rows that are equal
    to the largest share the attention, evenly."""
    top = 255.0 if dt == BF else 2047.0
    factors = [float(1 + (37 * j) % 201) for j in range(L)]
    for j in (0, L // 2, L - 1):                                      # early, late and last: three equal ones, or the only ones
        factors[j] = top
    if a < 0:
        factors = [-f for f in factors]
    m, q = steep_scores(dt, factors, a)
    assert float(abs(a) * 64 * scale) > 1000                          # a step of one factor: nothing is left of the others
    want = m.V[m.where(0, L)[0], :, m.where(0, L)[1]][[j for j in range(L) if abs(factors[j]) == top], 0].double()
    out, lse, weight, _ = call(m, q, None, None, scale)
    half = torch.finfo(dt).eps / 2
    mean, mass = want.mean(0), want.abs().mean(0)
    tol = half * mean.abs() + 2.0 ** -15 * mass + torch.finfo(dt).tiny
    assert torch.isfinite(out).all() and ((out.cpu().double()[0] - mean).abs() <= tol).all()
    exact = abs(float(q[0, 0, 0])) * top * 64 * float(torch.tensor(scale)) + math.log(len(want))
    assert ((lse.cpu().double() - exact).abs() <= (64 * 2.0 ** -23 + 2.0 ** -21) * exact).all()   # 64 products, summed by steps that may cut
    page, slot = (t.cuda() for t in m.where(0, L))
    gain = (weight - m.weight.float().cuda().nan_to_num(0.0))[page, 0, slot].cpu()
    equal = torch.tensor([abs(f) == top for f in factors])
    assert ((gain[equal] - 2.0 / len(want)).abs() <= 2.0 ** -20).all() and (gain[~equal] == 0).all()
