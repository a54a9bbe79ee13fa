"""Settings of a session that only some of a chunk's calls read."""
import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200.session import PagedCacheSession, PagedPoolSession
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


def rows_of(s, n):
    """What problem n holds, in order of its positions, per head: positions, weights, keys, values."""
    length, page = int(s.lens[n]), s.Kp.shape[2]
    r = torch.arange(max(length, 0), device="cuda")
    p, at = s.table[n].long()[r // page], r % page
    pos = s.pos[p, :, at]
    order = pos.argsort(0)
    pick = lambda t: t[p, :, at].gather(0, order[..., None].expand(-1, -1, t.shape[3]) if t.dim() == 4 else order)  # noqa: E731
    return pick(s.pos), pick(s.weight), pick(s.Kp), pick(s.Vp)


@pytest.mark.parametrize("interleaved", [False, True])
def test_steps_turned_by_the_caller_are_chunks_of_one_token(interleaved):
    """turn() and decode() against chunk() of one token: the same rows bit for bit, the same outputs but for what P and sums round."""
    freqs, factor = ec.ec_rotary_frequencies(64, scaling=ec.EC_ROTARY_BY_PARTS, stretch=4.0, trained=32.0)
    a, b = (PagedPoolSession(N=3, H=2, D=64, Hq=4, budget=200, recent=8, sinks=1, scale=0.125, pool_rows=900, chunk=90, page_size=16, rot=64,
                             interleaved=interleaved, freqs=freqs, factor=factor) for _ in range(2))
    q, k, v = rand((100, 4, 64), BF, 1).cuda(), rand((100, 2, 64), BF, 2).cuda(), rand((100, 2, 64), BF, 3).cuda()
    counts = torch.tensor([60, 0, 40], dtype=torch.int32, device="cuda")
    for s in (a, b):
        s.chunk(q, k, v, counts, torch.empty_like(q))
        s.end(1)
    ones = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    for step in range(5):
        q1, k1, v1 = (rand((3, h, 64), BF, 10 * step + h).cuda() for h in (4, 2, 3))
        v1 = v1[:, :2].contiguous()
        qt, kt, one = torch.empty_like(q1), torch.empty_like(k1), torch.empty_like(q1)
        a.turn(q1, qt)
        a.turn(k1, kt)
        a.decode(qt, kt, v1, one)
        on = torch.tensor([0, 2], device="cuda")
        many = torch.empty_like(q1[on])
        b.chunk(q1[on], k1[on], v1[on], ones, many)
        assert (one[1] == 0).all() and a.lens.tolist() == b.lens.tolist() == [61 + step, -1, 41 + step]
        assert a.seen.tolist()[0] == b.seen.tolist()[0] == 61 + step
        # values of about one, averaged: each rounds P (one of them in two parts) and the result, by half a step
        assert (one[on].float() - many.float()).abs().max() <= 4 * 2.0 ** -9 * v1.float().abs().max()
        for n in (0, 2):
            for x, y, exact in zip(rows_of(a, n), rows_of(b, n), (True, False, True, True)):
                assert torch.equal(x, y) if exact else torch.allclose(x, y, rtol=3e-5, atol=3e-5)
    assert a.status() == b.status() == ec.EC_OK


def test_rows_with_scores_join_a_pool_as_they_join_a_cache():
    """append() on a pool against PagedCacheSession's: the same rows stay; a problem without pages keeps what it had."""
    N, H, D, budget = 4, 2, 64, 48
    kw = dict(N=N, H=H, D=D, budget=budget, recent=4, sinks=1, scale=0.125, page_size=16)
    a, b = PagedPoolSession(**kw, pool_rows=9 * 16, chunk=16), PagedCacheSession(**kw)
    for call, counts in enumerate(([30, 40, 0, 16], [100, 5, 1, 0], [3, 3, 3, 3])):
        T = max(counts)
        K, V = rand((N, H, T, D), BF, 10 + call).cuda(), rand((N, H, T, D), BF, 20 + call).cuda()
        w = torch.rand(N, H, T, generator=torch.Generator().manual_seed(call)).cuda()
        c = torch.tensor(counts, dtype=torch.int32, device="cuda")
        a.append(K, V, w, c)
        granted = a.granted.tolist()
        assert granted == counts
        b.append(K, V, w, c)
        assert a.lens.tolist() == b.lens.tolist() and a.seen.tolist() == b.seen.tolist() and max(a.lens.tolist()) <= budget
        for n in range(N):
            for x, y in zip(rows_of(a, n), rows_of(b, n)):
                assert torch.equal(x, y)
    # 3 + 3 + 1 + 2 of nine pages are held: none is left for a problem that grows past its own
    assert int(a.pages.n_free) == 0
    before = [rows_of(a, n) for n in range(N)]
    K, w = rand((N, H, 20, D), BF, 30).cuda(), torch.ones(N, H, 20, device="cuda")
    a.append(K, K, w, torch.tensor([0, 0, 20, 2], dtype=torch.int32, device="cuda"))
    assert a.granted.tolist() == [0, 0, 0, 2] and a.lens.tolist() == [48, 48, 4, 21]
    for n in (0, 1, 2):
        for x, y in zip(rows_of(a, n), before[n]):
            assert torch.equal(x, y)
    assert a.status() == ec.EC_OK
