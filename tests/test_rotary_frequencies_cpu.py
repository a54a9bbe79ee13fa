"""Frequencies by parts: who keeps theirs, who is stretched."""
import math

import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200 import build as ecbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    ecbuild.build()


@pytest.mark.parametrize("rot", [16, 64, 128])
@pytest.mark.parametrize("base", [1.5, 100.0, 10000.0, 1e6])
@pytest.mark.parametrize("trained", [0.5, 3.0, 7.0, 100.0, 4096.0, 1e9])
@pytest.mark.parametrize("fast,slow", [(32.0, 1.0), (5.0, 5.0), (0.6, 0.3)])
def test_by_parts_goes_by_the_turns(rot, base, trained, fast, slow):
    """Pairs that turn more than `fast` times over `trained` positions keep their frequency, those that turn less than `slow` times get
    it divided by the stretch, those between lie between: also where all of them are on one side."""
    f, _ = ec.ec_rotary_frequencies(rot, base=base)
    g, _ = ec.ec_rotary_frequencies(rot, base=base, scaling=ec.EC_ROTARY_BY_PARTS, stretch=4.0, trained=trained, fast=fast, slow=slow)
    turns = trained * f / (2 * math.pi)
    keep, full = turns > fast * (1 + 1e-9), turns < slow * (1 - 1e-9)
    assert torch.equal(g[keep], f[keep]) and torch.allclose(g[full], f[full] / 4, rtol=1e-15, atol=0)
    assert ((g <= f) & (g >= f / 4 * (1 - 1e-15))).all()
    assert (g[1:] <= g[:-1]).all()
