"""Settings of a session that only some of a chunk's calls read."""
import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200.session import PagedPoolSession
from test_paged_gpu import BF, rand

pytestmark = pytest.mark.gpu
GOOD = dict(N=2, H=2, D=64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=400, chunk=40)


def run(**kw):
    s = PagedPoolSession(**{**GOOD, **kw})
    q = rand((50, 2, 64), BF, 1).cuda()
    out = torch.empty_like(q)
    s.chunk(q, q, q, torch.tensor([30, 20], dtype=torch.int32, device="cuda"), out)
    assert s.status() == ec.EC_OK and s.lens.tolist() == [30, 20]
    return out


def test_frequencies_that_nothing_turns_by():
    freqs, _ = ec.ec_rotary_frequencies(64)
    assert torch.equal(run(), run(rot=0, freqs=freqs))


def test_frequencies_out_of_something_wider():
    freqs, _ = ec.ec_rotary_frequencies(64)
    wide = torch.stack([freqs, freqs * 2], 1)
    for f in (wide[:, 0], wide[:, 0].float().cuda()):
        assert torch.equal(run(rot=64, freqs=f), run(rot=64, freqs=f.double().contiguous()))


def test_everything_for_what_is_kept():
    run(recent=60, sinks=4)


def test_sizes_that_no_step_could_take():
    with pytest.raises((ValueError, ec.EcError)):
        PagedPoolSession(**{**GOOD, "N": 65536, "H": 64, "Hq": 64 * 8, "budget": 1, "recent": 0, "sinks": 0, "chunk": 1, "pool_rows": 16,
                            "page_size": 16})
