"""Tokens of a chunk whose scores leave nothing."""
import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from test_chunk_gpu import mirror, pack
from test_paged_gpu import BF, HF, rand, scratch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("lens,counts", [([40], [20]), ([700, 300], [200, 300]), ([3000], [5])])
def test_scores_of_minus_infinity_on_values_that_are_not_finite(lens, counts, dt):
    """A token whose scores are all -inf comes out as zero: values are not looked at, whether every token of its tile sees them or not."""
    m = mirror(lens, 1, 64, 16, dt)
    inf = float("inf")
    for n, length in enumerate(lens):
        page, slot = m.where(n, length)
        for K, V in ((m.K, m.V), (m.dev["K"], m.dev["V"])):
            K[page, 0, slot] = 0.0
            K[page, 0, slot, 0] = -inf
            V[page[length - counts[n] // 2:], 0, slot[length - counts[n] // 2:], 7] = inf
            V[page[0], 0, slot[0], 9] = float("nan")
    starts, tokens = pack(counts)
    q = rand((tokens, 1, 64), dt, 4).abs() + 0.5
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 1))
    out, lse = torch.empty(tokens, 1, 64, dtype=dt, device="cuda"), torch.empty(tokens, 1, device="cuda")
    ec.ec_paged_chunk_attention(q.cuda(), starts.cuda(), torch.tensor(counts, dtype=torch.int32).cuda(), cache, 0.125, out, lse, ws)
    assert (out == 0).all() and (lse == -inf).all()
