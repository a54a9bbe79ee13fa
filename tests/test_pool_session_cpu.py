"""Settings that a chunk's calls would refuse, after its rows have joined, are refused where the session is made."""
import pytest
import torch

from paper_2407_18121_b200 import build as ecbuild
from paper_2407_18121_b200.session import PagedPoolSession

GOOD = dict(N=2, H=2, D=64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=400, chunk=40)
ONES = torch.ones(16, dtype=torch.float64)


@pytest.fixture(scope="module", autouse=True)
def built():
    ecbuild.build()


@pytest.mark.parametrize("bad", [
    dict(Hq=3), dict(Hq=1), dict(Hq=-2), dict(Hq=2 * 129), dict(H=1024, Hq=1024 * 65), dict(N=0), dict(N=65537), dict(H=0),
    dict(recent=60, sinks=5), dict(recent=65), dict(recent=-1), dict(sinks=-1), dict(budget=0), dict(budget=-5, recent=0, sinks=0),
    dict(pool_rows=0), dict(chunk=0), dict(page_size=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=1e-60), dict(scale=float("nan")),
    dict(scale=1e39), dict(decay=0.0), dict(decay=1e-60), dict(decay=1.0 + 1e-12), dict(decay=float("nan")), dict(factor=float("inf")),
    dict(factor=float("nan")), dict(factor=1e39), dict(rot=32), dict(rot=24, freqs=ONES[:12]), dict(rot=32, freqs=ONES[:8]),
    dict(rot=-16, freqs=ONES), dict(rot=128, freqs=torch.ones(64))])
def test_settings_that_are_refused(bad):
    with pytest.raises(ValueError):
        PagedPoolSession(**{**GOOD, **bad})
