"""Counts that are an output of the same call: several CTAs would read them while one writes."""
import ctypes as C

from paper_2407_18121_b200 import binding as ec
from test_chunk_cpu import pool
from test_paged_cpu import L, P, paged  # noqa: F401 (L is the fixture)


def test_counts_that_the_call_writes_are_refused(L):  # noqa: F811
    r, p = C.byref(paged()), C.byref(pool())
    a, b, c, d = (P + 0x1000 * i for i in range(1, 5))
    for starts, granted, slots, positions in ((P, b, c, d), (a, P, c, d), (a, b, P, d), (a, b, c, P)):
        assert L.ec_paged_reserve(r, p, P, 5000, 1, 0, starts, granted, slots, positions, None) == ec.EC_ERR_ARG
    assert L.ec_paged_reserve(r, p, P, 0, 0, 64, None, P, None, None, None) == ec.EC_ERR_ARG
