"""Sequences so long that a row's distance times the group passes 32 bits."""
import math

import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from test_paged_gpu import BF, rand, scratch, state_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,length,count", [(128, (1 << 24) + 4, 3), (128, (1 << 24) - 64, 3), (16, (1 << 27) + 20, 11), (33, (1 << 26) + 2, 1)])
def test_the_oldest_rows_of_a_long_sequence_gather(G, length, count):
    """All but the first and the last pages of one head's table are absent: the rows in front have to gather as any others do."""
    D, page = 64, 64
    pages = -(-length // page)
    present = [0, 1, pages // 2, pages - 2, pages - 1]
    table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
    table[0, present] = torch.tensor([3, 0, 4, 1, 2], dtype=torch.int32, device="cuda")
    K, V = rand((5, 1, page, D), BF, 1), rand((5, 1, page, D), BF, 2)
    weight = torch.rand(5, 1, page, generator=torch.Generator().manual_seed(3))
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens, w = one + length, weight.cuda()
    state = torch.empty(ec.ec_paged_state_bytes(1), dtype=torch.uint8, device="cuda")
    cache = ec.ec_paged_init(K.cuda(), V.cuda(), w, torch.zeros(5, 1, page, dtype=torch.int32, device="cuda"), table, lens, lens.clone(), state)
    q, scale, decay = rand((count, G, D), BF, 4), 0.125, 0.9
    ws = scratch(ec.ec_paged_chunk_workspace(cache, G))
    out, lse = torch.empty(count, G, D, dtype=BF, device="cuda"), torch.empty(count, G, device="cuda")
    counts = one + count
    ec.ec_paged_chunk_attention(q.cuda(), one, counts, cache, scale, out, lse, ws)
    ec.ec_paged_chunk_weights(q.cuda(), lse, one, counts, cache, scale, decay, ws)
    assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE          # of the absent pages
    # the definition, over the rows that are there
    order = torch.tensor([3, 0, 4, 1, 2])
    at = torch.cat([torch.arange(p * page, (p + 1) * page) for p in present])
    Kr, Vr = K[order, 0].reshape(-1, D).double(), V[order, 0].reshape(-1, D).double()
    x = torch.einsum("tgd,ld->tgl", q.double(), Kr) * scale
    ax = torch.einsum("tgd,ld->tgl", q.double().abs(), Kr.abs()) * scale
    sees = (at[None] <= (length - count + torch.arange(count))[:, None])[:, None]
    x = x.masked_fill(~sees, -math.inf)
    want_lse = torch.logsumexp(x, -1)
    # a score is off by D products of fp32 and the exponent's roundings, an exponential by 2^-17, see the chunk's other tests
    rel = D * 2.0 ** -23 * ax.amax() + 2.0 ** -17 + 2 * x.masked_fill(~sees, 0.0).abs().amax() * 2.0 ** -21 + (count * G + 700) * 2.0 ** -24
    assert ((lse.cpu().double() - want_lse).abs() <= 2 * rel).all()
    z = lse.cpu().double()[..., None]
    share = decay ** (count - 1 - torch.arange(count, dtype=torch.float64))
    gain = torch.einsum("t,tgl->l", share, torch.exp(x - z))
    old = weight[order, 0].reshape(-1).double()
    new = torch.where(at < length, decay ** count * old + gain, old)
    got = w.cpu()[order, 0].reshape(-1).double()
    assert (gain[:128] > 0.001).all()
    assert ((got - new).abs() <= 2 * rel * gain + 2.0 ** -22 * new).all(), f"worst by {float((got - new).abs().max()):.3g}"
    half = torch.finfo(BF).eps / 2
    p = torch.exp(x - want_lse[..., None])
    want, mass = torch.einsum("tgl,ld->tgd", p, Vr), torch.einsum("tgl,ld->tgd", p, Vr.abs())
    assert ((out.cpu().double() - want).abs() <= half * want.abs() + (half + 2 * rel) * mass * (1 + half)).all()
