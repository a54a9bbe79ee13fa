"""Attention over a paged cache where most rows lie far below the leading ones: what is left for them is the output."""
import math

import pytest
import torch

from paged_bounds import Exact
from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from test_paged_gpu import BF, HF, rand, scratch, state_of

pytestmark = pytest.mark.gpu


def call(m, q, k, v, scale, accumulate=True, decay=1.0):
    """The kernel's outputs, twice from the same state: they have to be the same bits."""
    cache = m.cache(ec)
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    ws = scratch(ec.ec_paged_attention_workspace(cache, q.shape[1], accumulate))
    before, got = m.dev["weight"].clone(), []
    for _ in range(2):
        m.dev["weight"].copy_(before)
        out = torch.full(q.shape, float("nan"), dtype=m.dtype, device="cuda")
        lse = torch.full(q.shape[:2], float("nan"), device="cuda")
        w_new = torch.full((m.N, m.H), float("nan"), device="cuda") if accumulate and k is not None else None
        ec.ec_paged_attention(up(q), up(k), up(v), cache, scale, accumulate, decay, out, lse, w_new, ws)
        torch.cuda.synchronize()
        got.append([out, lse, m.dev["weight"].clone(), w_new])
    for a, b in zip(*got):
        assert a is None or torch.equal(a.nan_to_num(77.0), b.nan_to_num(77.0)), "two runs differ"
    assert ec.ec_device_status(state_of(cache)) == ec.EC_OK
    return got[0]


def check(m, q, k, v, scale, decay=1.0):
    m.weight = m.dev["weight"].cpu().double()
    e = Exact(m, q, k, v, scale, decay)
    out, lse, weight, w_new = call(m, q, k, v, scale, True, decay)
    e.assert_out(out)
    e.assert_lse(lse)
    e.assert_weights(weight, w_new)
    return e


def leading_rows(m, n, rows, lead, q_unit, scale, value):
    """Every row of problem n scores 0 and has values near `value` but for `rows`, which lead by `lead` and have zeros."""
    page, slot = m.where(n, int(m.lens[n]))
    L, H, D = len(page), m.H, m.D
    V = value * (1 + 0.25 * torch.rand(L, H, D, generator=torch.Generator().manual_seed(L)))
    K = torch.zeros(L, H, D)
    V[rows] = 0.0
    K[rows, :, 0] = lead / (scale * q_unit)
    for pool, x in ((m.K, K), (m.V, V)):
        pool[page, :, slot] = x.to(m.dtype)
    m.dev["K"].copy_(m.K)
    m.dev["V"].copy_(m.V)


@pytest.mark.parametrize("dt", [HF, BF])
@pytest.mark.parametrize("lead", [8.0, 12.0, 16.0, 17.5, 20.0, 30.0])
@pytest.mark.parametrize("H,L,D,G", [(2, 8192, 64, 1), (2, 4096, 128, 4), (80, 2048, 64, 12), (600, 1024, 64, 1)])
def test_many_rows_far_below_a_leading_one(H, L, D, G, lead, dt):
    """A row that gathers the attention and has nothing to say: the output is what is left for the others, however little."""
    m = PagedMirror([L], H, D, 64, L, dt)
    scale, q_unit = 0.125, 8.0
    leading_rows(m, 0, torch.arange(0, 256, 16), lead, q_unit, scale, 4096.0)
    q = torch.zeros(1, H * G, D)
    q[:, :, 0] = q_unit
    k, v = torch.zeros(1, H, D, dtype=dt), rand((1, H, D), dt, 3)
    check(m, q.to(dt), k, v, scale)


@pytest.mark.parametrize("lead", [9.0, 14.0, 19.0])
def test_little_rows_beside_the_leading_one(lead):
    """The same within a few tiles: there is nobody else to make up for them."""
    for L, D in ((33, 64), (20, 128), (90, 128)):
        m = PagedMirror([L, L], 2, D, 16, 96, HF)
        for n in range(2):
            leading_rows(m, n, torch.tensor([0, L - 1]), lead, 8.0, 0.125, 8192.0)
        q = torch.zeros(2, 4, D)
        q[:, :, 0] = 8.0
        check(m, q.to(HF), None, None, 0.125)
