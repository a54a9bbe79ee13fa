"""Places of a running batch that sequences leave and others take."""
import pytest
import torch

from paged_bounds import Exact
from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200.session import PagedCacheSession
from test_paged_gpu import BF, HF, adopt, rand

pytestmark = pytest.mark.gpu


def steps(s, m, count, seed, recent, sinks):
    """Generation steps compared with the definition from the weights that the device holds."""
    N, H, D, Hq = s.N, s.H, s.D, s.Hq
    for i in range(count):
        q, k, v = (rand((N, h, D), m.dtype, seed + 3 * i + j) for j, h in enumerate((Hq, H, H)))
        out = torch.empty(N, Hq, D, dtype=m.dtype, device="cuda")
        m.weight = s.weight.cpu().double()
        e = Exact(m, q, k, v, s.scale, s.decay)
        s.decode(q.cuda(), k.cuda(), v.cuda(), out)
        e.assert_out(out, f"step {i}")
        tol = float(e.weight_tol.max()) + float(e.w_new_tol.max()) + 2.0 ** -24
        m.weight = e.weight
        m.append(k[:, :, None], v[:, :, None], e.w_new[:, :, None], None, None, 1, False, s.budget, recent, sinks)
        m.assert_same_rows(tol, f"step {i}")
    return m


@pytest.mark.parametrize("how", ["steps", "prompt"])
@pytest.mark.parametrize("dt", [BF, HF])
def test_a_place_that_is_taken_again_keeps_its_first_tokens(dt, how):
    N, H, D, budget, recent, sinks = 3, 2, 64, 24, 4, 3
    s = PagedCacheSession(N, H, D, budget, recent, sinks, 0.125, Hq=4, page_size=16, dtype=dt)
    K, V = (rand((N, H, 40, D), dt, i) for i in range(2))
    s.append(K.cuda(), V.cuda(), None, fresh=True)
    m = adopt(s)
    steps(s, m, 3, 100, recent, sinks)
    others = m.seen.clone()
    s.end(1)
    m.lens[1] = -1
    assert s.lens.tolist() == [budget, -1, budget]
    steps(s, m, 2, 200, recent, sinks)
    s.begin(1)
    m.lens[1] = m.seen[1] = 0
    assert s.lens.tolist() == [budget, 0, budget] and s.seen.tolist() == [others[0] + 2, 0, others[2] + 2]
    if how == "prompt":                          # its prompt alone, in pieces, while the others stay as they are
        for i, T in enumerate((20, 15)):
            K, V, w = (rand((N, H, T, D), dt, 40 + 4 * i + j) for j in range(3))
            w = w[..., 0].float().abs()
            counts = torch.tensor([0, T, 0], dtype=torch.int32)
            m.weight = s.weight.cpu().double()
            s.append(K.cuda(), V.cuda(), w.cuda(), counts.cuda())
            m.append(K, V, w, None, counts, T, False, budget, recent, sinks)
            m.assert_same_rows(0.0, "prompt")
    steps(s, m, budget + 8, 300, recent, sinks)
    page, slot = m.where(1, budget)
    for h in range(H):
        held = s.pos.cpu()[page, h, slot]
        assert {0, 1, 2} <= set(held.tolist())   # the sequence's own first tokens
    assert s.status() == ec.EC_OK


def test_places_are_looked_over():
    s = PagedCacheSession(2, 1, 64, 32, 4, 1, 0.125)
    s.lens.fill_(5)
    s.seen.fill_(9)
    for call in (s.begin, s.end):
        for bad in (-1, 2, 1.0, True, None):
            with pytest.raises((ValueError, TypeError)):
                call(bad)
    assert s.lens.tolist() == [5, 5] and s.seen.tolist() == [9, 9]


def test_a_place_begins_and_ends_in_stream_order():
    """Also inside a captured graph: the replay begins the place anew."""
    s = PagedCacheSession(2, 1, 64, 32, 4, 1, 0.125)
    q, k, v = (rand((2, 1, 64), BF, i).cuda() for i in range(3))
    out = torch.empty_like(q)
    s.decode(q, k, v, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.begin(0)
        s.decode(q, k, v, out)
        s.decode(q, k, v, out)
    for n in range(3):
        graph.replay()
    assert s.lens.tolist() == [2, 7] and s.seen.tolist() == [2, 7] and s.pos[0, 0, :2].tolist() == [0, 1]
