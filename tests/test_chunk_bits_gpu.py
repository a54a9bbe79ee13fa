"""The bits of a chunk's attention are its own: what lies in rows that are nobody's does not reach them."""
import math

import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from test_chunk_gpu import mirror, pack
from test_paged_gpu import BF, HF, rand, scratch

pytestmark = pytest.mark.gpu


def attend(m, q, starts, counts, G):
    cache = m.cache(ec)
    tokens = q.shape[0]
    out = torch.full((tokens, m.H * G, m.D), 7.0, dtype=m.dtype, device="cuda")
    lse = torch.full((tokens, m.H * G), 7.0, device="cuda")
    ws = scratch(ec.ec_paged_chunk_workspace(cache, m.H * G))
    ec.ec_paged_chunk_attention(q, starts, counts, cache, 1.0 / math.sqrt(m.D), out, lse, ws)
    return out, lse


def assert_same_bits(a, b, rows, what):
    for x, y, name in zip(a, b, ("out", "lse")):
        assert not torch.isnan(x[rows]).any() and (x[rows] < math.inf).all(), f"{what}: {name}"   # -inf: a token that sees nothing
        assert torch.equal(x[rows], y[rows]), f"{what}: {name} differs by {float((x[rows].float() - y[rows].float()).abs().max()):.3g}"


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 7, 16])
def test_packed_rows_of_nobody_and_of_others(G, D, dt):
    """A tile that is not full holds the rows that come next in the packed queries."""
    lens, counts, gap = [700, 300, 129, 2000], [max(1, 40 // G), 5, max(1, 200 // G), 1], 130 // G + 1
    m = mirror(lens, 2, D, 16, dt)
    starts, tokens = pack(counts, gap)
    mine = torch.zeros(tokens, dtype=torch.bool)
    for s, c in zip(starts.tolist(), counts):
        mine[s:s + c] = True
    sd, cd = starts.cuda(), torch.tensor(counts, dtype=torch.int32).cuda()
    q = rand((tokens, 2 * G, D), dt, 3)
    q[~mine] = 0.0
    want = attend(m, q.cuda(), sd, cd, G)
    for fill in (float("nan"), float("inf"), 1000.0, -1000.0):
        q[~mine] = fill
        assert_same_bits(attend(m, q.cuda(), sd, cd, G), want, mine, f"rows of nobody = {fill}")
    starts, tokens = pack(counts)                              # the next problem's rows are next to one's own
    q = rand((tokens, 2 * G, D), dt, 3)
    first = torch.arange(tokens) < counts[0]
    sd = starts.cuda()
    want = attend(m, q.cuda(), sd, cd, G)
    for fill in (float("nan"), 1000.0, 0.0):
        q[~first] = fill
        assert_same_bits(attend(m, q.cuda(), sd, cd, G), want, first, f"the next problem's queries = {fill}")


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [3, 5, 7, 12, 33, 100])
def test_rows_of_a_tile_that_no_copy_fills(G, D, dt):
    """Where the group does not divide 128 the tile's last rows hold what an earlier kernel left there."""
    per = 128 // G
    lens, counts = [900, 650, 400], [2 * per, per, max(1, per // 2)]
    m = mirror(lens, 2, D, 16, dt)
    starts, tokens = pack(counts)
    sd, cd = starts.cuda(), torch.tensor(counts, dtype=torch.int32).cuda()
    q = rand((tokens, 2 * G, D), dt, 4).cuda()
    before = mirror([256] * 300, 1, D, 64, dt)
    bs, n = pack([256] * 300)
    bs, bc = bs.cuda(), torch.full((300,), 256, dtype=torch.int32, device="cuda")
    results = []
    for fill in (0.0, float("nan"), 1000.0):
        attend(before, torch.full((n, 1, D), fill, dtype=dt, device="cuda"), bs, bc, 1)
        results.append(attend(m, q, sd, cd, G))
    rows = torch.ones(tokens, dtype=torch.bool)
    for r, what in zip(results[1:], ("not a number", "large")):
        assert_same_bits(r, results[0], rows, what)
