"""Attention over a paged cache within tolerances that follow from its roundings, element by element: outputs, normalisers,
and what every row gains."""
import math

import pytest

from paged_reference import PagedMirror
from test_paged_bounds_cpu import CASES, inputs
from test_paged_gpu import BF, HF, rand
from test_paged_precision_gpu import check

pytestmark = pytest.mark.gpu


def on_device(m):
    m.dev = {k: t.to("cuda") for k, t in dict(K=m.K, V=m.V, weight=m.weight.float(), pos=m.pos, table=m.table, lens=m.lens,
                                              seen=m.seen).items()}
    return m


@pytest.mark.parametrize("decay", [1.0, 0.5])
@pytest.mark.parametrize("case", CASES)
def test_where_a_rounding_of_p_would_show(case, decay):
    m, q, k, v, scale = inputs(case)
    check(on_device(m), q, k, v, scale, decay)


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("lens,H,D,G,page,cap", [([20000], 1, 64, 4, 64, 20000), ([1000, 333, 666], 40, 64, 1, 64, 1000),
                                                 ([130, 65, 1, 0, -1] * 13, 16, 64, 1, 16, 130), ([700, 20], 2, 128, 33, 24, 720),
                                                 ([40, 300], 3, 128, 2, 4, 9000)])
def test_what_every_row_gains(lens, H, D, G, page, cap, dt):
    """Also a table that reaches much further than the rows."""
    m = PagedMirror(lens, H, D, page, cap, dt)
    q, k, v = (rand((len(lens), h, D), dt, 30 + i) for i, h in enumerate((H * G, H, H)))
    check(m, q, k, v, 1.0 / math.sqrt(D), 0.75)
