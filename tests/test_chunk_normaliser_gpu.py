"""The weights of a chunk go by the normaliser that they are given, and by nothing else of a token that takes no part."""
import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from test_chunk_gpu import mirror, pack
from test_paged_gpu import BF, HF, rand, scratch, state_of

pytestmark = pytest.mark.gpu


def gather(m, q, lse, starts, counts, decay=1.0, scale=0.125):
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, q.shape[1]))
    ec.ec_paged_chunk_weights(q.cuda(), lse.cuda(), starts.cuda(), torch.tensor(counts, dtype=torch.int32).cuda(), cache, scale, decay, ws)
    assert ec.ec_device_status(state_of(cache)) == ec.EC_OK
    return m.dev["weight"].clone()


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("G", [1, 3, 4])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_token_without_a_normaliser_takes_no_part(bad, G, dt):
    """-inf leaves a token out, whatever its query holds."""
    lens, counts = [700, 90], [200, 90]
    starts, tokens = pack(counts)
    q = rand((tokens, 2 * G, 64), dt, 2)
    lse = torch.full((tokens, 2 * G), 6.0)
    out = torch.tensor([0, 1, 31, 77, 199, 200, 289])
    lse[out] = -float("inf")
    results = []
    for fill in (0.0, bad):
        q[out] = fill
        m = mirror(lens, 2, 64, 16, dt)
        results.append(gather(m, q, lse, starts, counts, 0.99))
    for n, rows in enumerate(lens):
        page, slot = m.where(n, rows)
        a, b = (r.cpu()[page, :, slot] for r in results)
        assert torch.isfinite(a).all() and torch.equal(a, b)
