"""Host-side checks of the chunk's entry points: refusals, workspace sizes, frequencies, and the plain forms against hand-worked cases."""
import ctypes as C
import math

import pytest
import torch

from chunk_reference import ChunkExact, PoolModel, rotary
from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from test_paged_cpu import BAD, L, P, paged  # noqa: F401 (L is the fixture)

BIG = 1 << 40


def pool(**kw):
    p = ec._ec_pages()
    v = dict(free_pages=P, n_free=P, held=P)
    v.update(kw)
    for k, x in v.items():
        setattr(p, k, x)
    return p


@pytest.mark.parametrize("bad,status", BAD)
def test_a_bad_description_is_refused_everywhere(L, bad, status):  # noqa: F811
    r, p = C.byref(paged(**bad)), C.byref(pool())
    assert L.ec_paged_release(r, p, None) == status
    assert L.ec_paged_reserve(r, p, P, 4, 1, 0, P, P, P, P, None) == status
    assert L.ec_paged_join(P, 512, 64, P, 512, 64, P, 512, 64, P, 512, 64, None, P, P, r, 6, 4, P, 32, 0, 1.0, None) == status
    assert L.ec_paged_chunk_attention(P, 512, 64, P, P, r, 6, 4, 1.0, P, 512, 64, None, P, BIG, None) == status
    assert L.ec_paged_chunk_weights(P, 512, 64, P, P, P, r, 6, 4, 1.0, 1.0, P, BIG, None) == status
    assert L.ec_paged_chunk_workspace(r, 6) == 0


def test_attention_and_weights_refusals(L):  # noqa: F811
    r = C.byref(paged())

    def a(q=P, qt=512, qh=64, s=P, c=P, Hq=6, tokens=4, scale=1.0, out=P, ot=512, oh=64, lse=None, ws=P, size=BIG, decay=1.0, which=0):
        if which:
            return L.ec_paged_chunk_weights(q, qt, qh, lse, s, c, r, Hq, tokens, scale, decay, ws, size, None)
        return L.ec_paged_chunk_attention(q, qt, qh, s, c, r, Hq, tokens, scale, out, ot, oh, lse, ws, size, None)
    for which in (0, 1):
        z = P if which else None
        assert a(q=None, lse=z, which=which) == 1 and a(s=None, lse=z, which=which) == 1 and a(c=None, lse=z, which=which) == 1
        assert a(Hq=7, lse=z, which=which) == 2 and a(Hq=0, lse=z, which=which) == 2 and a(Hq=3 * 129, lse=z, which=which) == 2
        assert a(tokens=-1, lse=z, which=which) == 2 and a(tokens=1 << 30, lse=z, which=which) == 2
        for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
            assert a(scale=scale, lse=z, which=which) == 4
        assert a(q=P + 8, lse=z, which=which) == 3 and a(s=P + 2, lse=z, which=which) == 3 and a(lse=P + 2, which=which) == 3
        assert a(qt=511, lse=z, which=which) == 4 and a(qh=60, lse=z, which=which) == 4 and a(qh=32, lse=z, which=which) == 4
        assert a(qt=0, lse=z, which=which) == 4 and a(qt=-512, lse=z, which=which) == 4
        assert a(ws=None, lse=z, which=which) == 5 and a(size=L.ec_paged_chunk_workspace(r, 6) - 1, lse=z, which=which) == 5
        assert a(ws=P + 64, lse=z, which=which) == 3
        assert a(tokens=0, lse=z, which=which) == 0                                             # nothing to do
    assert a(out=None) == 1 and a(out=P + 8) == 3 and a(oh=60) == 4
    assert a(which=1) == 1                                                                      # the normaliser is needed
    for decay in (0.0, 1.5, float("nan")):
        assert a(lse=P, decay=decay, which=1) == 4
    assert L.ec_paged_chunk_workspace(r, 7) == 0 and L.ec_paged_chunk_workspace(None, 6) == 0


def test_reserve_release_and_join_refusals(L):  # noqa: F811
    r, p = C.byref(paged()), C.byref(pool())
    assert L.ec_paged_release(r, None, None) == 1 and L.ec_paged_release(r, C.byref(pool(held=None)), None) == 1
    assert L.ec_paged_release(r, C.byref(pool(n_free=P + 2)), None) == 3
    f = L.ec_paged_reserve
    assert f(r, p, None, 4, 1, 0, P, P, P, P, None) == 1 and f(r, p, P, 4, 1, 0, P, None, P, P, None) == 1
    assert f(r, p, P, -1, 1, 0, P, P, P, P, None) == 4 and f(r, p, P, 4, 0, -1, P, P, None, None, None) == 4
    assert f(r, p, P, 4, 0, 0, P, P, P, None, None) == 4                                        # slots of rows that do not join
    assert f(r, p, P + 1, 4, 1, 0, P, P, P, P, None) == 3
    assert f(C.byref(paged(N=1 << 17, H=1)), p, P, 4, 1, 0, P, P, P, P, None) == 2
    g = L.ec_paged_join

    def j(q=P, qo=P, k=P, v=P, w=None, s=P, pos=P, Hq=6, tokens=4, fr=P, rot=32, inter=0, factor=1.0, kt=512, kh=64):
        return g(q, 512, 64, qo, 512, 64, k, kt, kh, v, 512, 64, w, s, pos, r, Hq, tokens, fr, rot, inter, factor, None)
    assert j(k=None) == 1 and j(v=None) == 1 and j(s=None) == 1 and j(pos=None) == 1 and j(q=None) == 1 and j(qo=None) == 1
    assert j(Hq=0) == 1 and j(fr=None) == 1                                                     # queries without heads; turns without frequencies
    assert j(rot=24) == 4 and j(rot=12, inter=1) == 4 and j(rot=128) == 4 and j(rot=-16) == 4 and j(factor=float("inf")) == 4
    assert j(kt=100) == 4 and j(kh=32) == 4 and j(k=P + 8) == 3 and j(w=P + 2) == 3 and j(fr=P + 4) == 3
    assert j(tokens=-1) == 2 and j(Hq=-1) == 2 and j(tokens=0) == 0


def test_rotary_refusals(L):  # noqa: F811
    def f(x=P, xt=512, xh=64, out=P, pos=P, fr=P, N=2, T=3, heads=4, D=64, dt=0, rot=64, inter=0, factor=1.0, xn=4096, pn=3):
        return L.ec_rotary(x, xn, xt, xh, out, 4096, 512, 64, pos, pn, fr, N, T, heads, D, dt, rot, inter, factor, 0, None)
    assert f(x=None) == 1 and f(out=None) == 1 and f(pos=None) == 1 and f(fr=None) == 1
    assert f(D=96) == 2 and f(N=-1) == 2 and f(T=-1) == 2 and f(heads=0) == 2 and f(N=1 << 16, T=1 << 16) == 2
    assert f(dt=2) == 4 and f(rot=40) == 4 and f(rot=20, inter=1) == 4 and f(rot=80) == 4 and f(factor=float("nan")) == 4
    assert f(xt=511) == 4 and f(xh=32) == 4 and f(xn=-8) == 4 and f(pn=-1) == 4 and f(x=P + 8) == 3 and f(pos=P + 2) == 3
    assert f(N=0) == 0 and f(T=0) == 0


def test_no_tokens_are_nothing_to_do(L):  # noqa: F811
    """Tensors without elements have no address."""
    r = C.byref(paged())
    size = L.ec_paged_chunk_workspace(r, 6)
    assert L.ec_paged_chunk_attention(None, 384, 64, P, P, r, 6, 0, 1.0, None, 384, 64, None, P, size, None) == 0
    assert L.ec_paged_chunk_weights(None, 384, 64, None, P, P, r, 6, 0, 1.0, 1.0, P, size, None) == 0
    assert L.ec_paged_join(None, 384, 64, None, 384, 64, None, 128, 64, None, 128, 64, None, None, None, r, 6, 0, P, 32, 0, 1.0, None) == 0
    assert L.ec_rotary(None, 0, 256, 64, None, 0, 256, 64, None, 0, P, 2, 0, 4, 64, 0, 64, 0, 1.0, 0, None) == 0
    assert L.ec_paged_join(None, 384, 64, None, 384, 64, None, 128, 64, None, 128, 64, None, None, None, r, 6, 0, P, 24, 0, 1.0, None) == 4


def test_the_arrays_of_a_pool_stay():
    t = torch.zeros(3, dtype=torch.int32)
    pages = ec.ec_pages(t, t, t)
    for name in ("free_pages", "n_free", "held"):
        assert getattr(pages, name) is t
        with pytest.raises(AttributeError):
            setattr(pages, name, t.clone())


def test_frequencies(L):  # noqa: F811
    f, factor = ec.ec_rotary_frequencies(64)
    assert factor == 1.0 and torch.allclose(f, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32), rtol=1e-15, atol=0)
    g, _ = ec.ec_rotary_frequencies(64, scaling=ec.EC_ROTARY_LINEAR, stretch=4.0)
    assert torch.allclose(g, f / 4, rtol=1e-15, atol=0)
    g, _ = ec.ec_rotary_frequencies(64, scaling=ec.EC_ROTARY_BASE, stretch=4.0)
    # the slowest pair is stretched in full, the fastest not at all
    assert g[0] == 1.0 and math.isclose(float(g[31]), float(f[31]) / 4, rel_tol=1e-12)
    g, factor = ec.ec_rotary_frequencies(128, scaling=ec.EC_ROTARY_BY_PARTS, stretch=8.0, trained=4096.0)
    f, _ = ec.ec_rotary_frequencies(128)
    assert math.isclose(factor, 0.1 * math.log(8.0) + 1.0, rel_tol=1e-6)
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns > 40], f[turns > 40]) and torch.allclose(g[turns < 0.9], f[turns < 0.9] / 8, rtol=1e-15, atol=0)
    assert ((g <= f) & (g >= f / 8)).all()
    for kw in (dict(rot=0), dict(rot=7), dict(rot=2048), dict(rot=64, base=1.0), dict(rot=64, base=float("nan")), dict(rot=64, scaling=4),
               dict(rot=64, scaling=1, stretch=0.5), dict(rot=2, scaling=2, stretch=2.0), dict(rot=64, scaling=3, stretch=2.0),
               dict(rot=64, scaling=3, stretch=2.0, trained=4096.0, fast=1.0, slow=2.0)):
        with pytest.raises(ec.EcError):
            ec.ec_rotary_frequencies(**kw)


def test_the_plain_rotary_by_hand():
    x = torch.tensor([[[1.0, 0.0, 5.0, 6.0]]])
    quarter = torch.tensor([math.pi / 2], dtype=torch.float64)
    assert torch.allclose(rotary(x, torch.tensor([1]), quarter, 2.0, 2, True), torch.tensor([[[0.0, 2.0, 5.0, 6.0]]], dtype=torch.float64), atol=1e-12)
    assert torch.allclose(rotary(x, torch.tensor([1]), quarter, 1.0, 2, True, True), torch.tensor([[[0.0, -1.0, 5.0, 6.0]]], dtype=torch.float64), atol=1e-12)
    y = torch.tensor([[[1.0, 2.0, 3.0, 4.0]]])
    two = torch.tensor([math.pi / 2, math.pi], dtype=torch.float64)
    assert torch.allclose(rotary(y, torch.tensor([1]), two, 1.0, 4, False), torch.tensor([[[-3.0, -2.0, 1.0, -4.0]]], dtype=torch.float64), atol=1e-12)


def test_the_plain_chunk_against_a_library_softmax():
    m = PagedMirror([7, 5], 2, 64, 4, 8, torch.float32, device=None)
    m.weight = m.weight.double()
    q = torch.randn(8, 4, 64, generator=torch.Generator().manual_seed(1))
    r = ChunkExact(m, q, torch.tensor([0, 3]), torch.tensor([3, 5]), 0.2, 0.5)
    for n, (start, cnt, length) in enumerate(((0, 3, 7), (3, 5, 5))):
        p, s = m.where(n, length)
        for t in range(cnt):
            upto = length - cnt + t + 1
            for i in range(4):
                x = (m.K[p, i // 2, s].double()[:upto] @ q[start + t, i].double()) * 0.2
                w = torch.softmax(x, 0)
                assert torch.allclose(r.out[start + t, i], w @ m.V[p, i // 2, s].double()[:upto], atol=1e-12)
                assert math.isclose(float(r.lse[start + t, i]), float(torch.logsumexp(x, 0)), rel_tol=1e-12)


def test_a_rounding_of_the_score_or_a_dropped_token_falls_outside_of_the_tolerance():
    """What the tolerances would show: the mask off by one row, and a token whose weight is left out."""
    m = PagedMirror([40], 1, 64, 8, 40, torch.bfloat16, device=None)
    q = torch.randn(20, 1, 64, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    good = ChunkExact(m, q, torch.tensor([0]), torch.tensor([20]), 0.125, 0.9)
    m.lens[0] = 39
    off = ChunkExact(m, q, torch.tensor([0]), torch.tensor([20]), 0.125, 0.9)
    with pytest.raises(AssertionError):
        good.assert_out(off.out)
    m.lens[0] = 40
    part = ChunkExact(m, q[:19], torch.tensor([0]), torch.tensor([19]), 0.125, 0.9)
    with pytest.raises(AssertionError):
        good.assert_weights(part.weight)


def test_the_pool_model_by_hand():
    m = PoolModel([5, -1, 3], [5, 9, 30], [2, 1, 2], [[0, 1, -1], [2, -1, -1], [3, 4, -1]], [5, 6], 4)
    m.release()                                   # problem 1 is over, problem 2 needs one page of its two
    assert m.free == [5, 6, 2, 4] and m.held == [2, 0, 1]
    starts, granted, slots, positions = m.reserve([4, 2, 2], 8)
    assert starts == [0, 4, 6, 8] and granted == [4, 0, 2]
    assert m.table[0] == [0, 1, 4] and m.table[2][:2] == [3, 2] and m.free == [5, 6]
    assert slots == [5, 6, 7, 16, -1, -1, 15, 8] and positions == [5, 6, 7, 8, -1, -1, 30, 31]
    assert m.lens == [9, -1, 5]
