"""The weights of a chunk go by the normaliser that they are given, and by nothing else of a token that takes no part."""
import math

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


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_the_exponent_is_rounded_once(sign):
    """One row a head and a score of zero: the gain is exp(-lse). The exponent, -lse log2(e), lies between 2^5 and 2^7 and is rounded by
    half a step, 2^-18 at most; the exponential is off by 2^-22 and the weight's sum rounded once."""
    H = 256
    m = mirror([1], H, 64, 16)
    m.dev["weight"].zero_()
    lse = sign * torch.linspace(40.0, 85.0, H)[None]
    weight = gather(m, torch.zeros(1, H, 64, dtype=BF), lse, torch.tensor([0], dtype=torch.int32), [1])
    page, slot = m.where(0, 1)
    got = weight.cpu()[page[0], :, slot[0]].double()
    off = (got / torch.exp(-lse[0].double()) - 1).abs()
    assert (off <= math.log(2.0) * 2.0 ** -18 + 2.0 ** -21).all(), float(off.max())


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
