"""The paged cache on the GPU against plain 64-bit forms: attention of one token with gathered weights, append with
eviction by weight, whole steps."""
import math

import numpy as np
import pytest
import torch

from paged_reference import PagedMirror, attention_bounds
from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200.session import PagedCacheSession

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def scratch(n):
    return torch.full((max(int(n), 256),), 0xA5, dtype=torch.uint8, device="cuda")


def rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def check_attention(m, G, new=True, accumulate=False, decay=1.0, scale=None, seed=1, q=None, drop=(), twice=True):
    N, H, D, dt = m.N, m.H, m.D, m.dtype
    scale = scale or 1.0 / math.sqrt(D)
    q = rand((N, H * G, D), dt, seed) if q is None else q
    k, v = (rand((N, H, D), dt, seed + 1), rand((N, H, D), dt, seed + 2)) if new else (None, None)
    cache = m.cache(ec)
    before = m.dev["weight"].clone()
    m.weight = before.cpu().double()             # a call before this one left fp32 weights: the definition starts from those
    old = m.weight.clone()
    ref, mass, dx = m.attention(q, k, v, scale, accumulate, decay, drop)
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    ws = scratch(ec.ec_paged_attention_workspace(cache, H * G, accumulate))
    results = []
    for _ in range(2 if twice else 1):
        m.dev["weight"].copy_(before)
        out = torch.full((N, H * G, D), float("nan"), dtype=dt, device="cuda")
        lse = torch.full((N, H * G), float("nan"), device="cuda")
        w_new = torch.full((N, H), float("nan"), device="cuda") if accumulate and new else None
        ec.ec_paged_attention(up(q), up(k), up(v), cache, scale, accumulate, decay, out, lse, w_new, ws)
        torch.cuda.synchronize()
        results.append([t.clone() for t in (out, lse, w_new, m.dev["weight"]) if t is not None])
    if twice:
        for a, b in zip(*results):
            assert torch.equal(a.nan_to_num(77.0), b.nan_to_num(77.0)), "two runs differ"
    out_tol, lse_tol, w_tol = attention_bounds(ref, mass, dx, dt, G)
    got = out.cpu().double()
    assert torch.isfinite(got).all()
    over = (got - ref[0]).abs() - out_tol
    assert (over <= 0).all(), f"out: {float(over.max()):.3g} over its tolerance"
    got = lse.cpu().double()
    empty = torch.isinf(ref[1])
    assert torch.equal(torch.isinf(got), empty)
    assert ((got - ref[1]).abs()[~empty] <= lse_tol[~empty]).all()
    if accumulate:
        # the row's old weight, its decay and the sum are rounded once each
        held = torch.isfinite(old)
        atol = w_tol + float(old[held].abs().max() if held.any() else 0.0) * 2.0 ** -22
        m.assert_same_rows(atol, "weights")
        if new:
            assert ((w_new.cpu().double() - ref[2]).abs() <= w_tol).all()
    else:
        m.assert_same_rows(0.0, "cache")
    if not drop:
        assert ec.ec_device_status(state_of(cache)) == ec.EC_OK
    return cache


def state_of(cache):
    return cache._tensors[-1]


EDGE = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, -1, 200]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("G", [1, 3, 8, 9, 16, 20])
def test_attention_edges_of_length_and_group(G, dt, D):
    check_attention(PagedMirror(EDGE, 2, D, 16, 208, dt, G=G), G, accumulate=True)


@pytest.mark.parametrize("G,accumulate", [(33, True), (128, False), (128, True)])
def test_attention_wide_groups(G, accumulate):
    check_attention(PagedMirror([70, 0, 300], 2, 64, 16, 304, G=G), G, accumulate=accumulate)


def test_attention_cuts_a_length_past_the_table():
    m = PagedMirror([96, 40], 2, 64, 32, 96)
    m.dev["lens"][0] = 5000
    cache = m.cache(ec)
    q = rand((2, 2, 64), BF, 1).cuda()
    outs = []
    for n in (5000, 96):
        m.dev["lens"][0] = n
        out = torch.empty_like(q)
        ws = scratch(ec.ec_paged_attention_workspace(cache, 2, False))
        ec.ec_paged_attention(q, None, None, cache, 0.125, False, 1.0, out, None, None, ws)
        torch.cuda.synchronize()
        outs.append(out)
        assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE      # from the first call on
    assert torch.equal(*outs)


@pytest.mark.parametrize("page", [1, 5, 16, 24, 64, 300])
@pytest.mark.parametrize("rows", ["heads", "tokens"])
def test_attention_pages_and_strides(page, rows):
    check_attention(PagedMirror([257, 3, 100], 3, 128, page, 300, rows=rows), 4, accumulate=True)


@pytest.mark.parametrize("new", [True, False])
@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("lens", [[0], [1], [0, 5, -1], [-1, -1], [700], [40, 3000, 9, 1500]])
def test_attention_with_and_without_the_own_row(lens, accumulate, new):
    check_attention(PagedMirror(lens, 2, 64, 32, 3008), 5, new=new, accumulate=accumulate)


@pytest.mark.parametrize("N,H,G,L", [(64, 16, 1, 130), (300, 4, 2, 70), (1, 1, 4, 20000), (3, 40, 1, 1000)])
def test_attention_many_units_and_long_rows(N, H, G, L):
    lens = [max(1, (L * (n % 7 + 1)) // 7) for n in range(N)]
    check_attention(PagedMirror(lens, H, 64, 64, L), G, accumulate=True, decay=0.75)


def test_attention_weights_decay():
    check_attention(PagedMirror([90, 400], 2, 128, 16, 400), 3, accumulate=True, decay=0.5)


def test_attention_rows_whose_score_is_minus_infinity():
    m = PagedMirror([100, 40], 2, 64, 16, 112)
    q = rand((2, 4, 64), BF, 3).abs() + 0.1
    p, s = m.where(0, 100)
    for pool in (m.K, m.dev["K"]):
        pool[p[10:90], :, s[10:90]] = -math.inf                       # every query sees -inf there
    check_attention(m, 2, q=q, accumulate=True)
    p, s = m.where(1, 40)
    for pool in (m.K, m.dev["K"]):
        pool[p, :, s] = -math.inf                                     # nothing but the own row is left of problem 1
    check_attention(m, 2, q=q, accumulate=True)
    check_attention(m, 2, q=q, new=False)                             # and here nothing at all


def test_attention_peaked_rows_and_large_scores():
    m = PagedMirror([900], 1, 128, 64, 960)
    for pool in (m.K, m.dev["K"]):
        for r, f in ((5, 4.0), (700, 9.0), (899, 16.0)):              # the running maximum rises late
            p, s = m.where(0, 900)
            pool[p[r], 0, s[r]] *= f
    check_attention(m, 4, scale=0.5, accumulate=True)


def test_attention_refuses_bad_pages_in_the_kernel():
    m = PagedMirror([100, 60], 2, 64, 16, 112)
    m.dev["table"][0, 2] = -1                                         # rows 32..47 of problem 0
    m.dev["table"][1, 3] = 1 << 30                                    # rows 48..59 of problem 1
    drop = {(0, j) for j in range(32, 48)} | {(1, j) for j in range(48, 60)}
    cache = check_attention(m, 2, accumulate=True, drop=drop)
    assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE
    assert ec.ec_device_status(state_of(m.cache(ec))) == ec.EC_OK   # a new description starts clean


# ---------------------------------------------------------------------------------------- append

def check_append(m, T, budget, recent=0, sinks=0, w=None, pos=None, counts=None, fresh=False, seed=4):
    N, H, D, dt = m.N, m.H, m.D, m.dtype
    K, V = (rand((N, H, T, D), dt, seed), rand((N, H, T, D), dt, seed + 1)) if T else (None, None)
    m.append(K, V, w, pos, counts, T, fresh, budget, recent, sinks)
    cache = m.cache(ec)
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    ws = scratch(ec.ec_paged_append_workspace(cache, T, budget))
    ec.ec_paged_append(up(K), up(V), up(w), up(pos), up(counts), cache, fresh, budget, recent, sinks, ws)
    torch.cuda.synchronize()
    m.assert_same_rows(0.0, "append")
    assert ec.ec_device_status(state_of(cache)) == ec.EC_OK


@pytest.mark.parametrize("T", [1, 3, 16, 17, 100])
@pytest.mark.parametrize("dt,D,rows", [(BF, 128, "heads"), (HF, 64, "tokens")])
def test_append_evicts_by_weight(T, dt, D, rows):
    N, H = 6, 3
    m = PagedMirror([120, 119, 60, 0, -1, 5], H, D, 16, 120, dt, rows)
    w = torch.rand(N, H, T, generator=torch.Generator().manual_seed(9))
    check_append(m, T, 120, recent=8, sinks=2, w=w)
    check_append(m, T, 120, recent=min(T, 100), sinks=4, w=w, counts=torch.tensor([T, 0, T // 2, 1, T, T + 9], dtype=torch.int32))


@pytest.mark.parametrize("kind", ["equal", "none", "coarse", "special"])
@pytest.mark.parametrize("T", [2, 40])
def test_append_equal_weights_and_special_values(kind, T):
    N, H, L = 2, 2, 300
    m = PagedMirror([L, L - 7], H, 64, 24, L)
    g = torch.Generator().manual_seed(5)
    w = None if kind == "none" else torch.randint(0, 3, (N, H, T), generator=g).float()
    if kind == "equal":
        w = torch.zeros(N, H, T)
    if kind == "special":
        w[:, :, 0], w[:, :, 1] = math.nan, -0.0
    for n in range(N):
        p, s = m.where(n, int(m.lens[n]))
        fill = torch.randint(0, 3, (len(p), H), generator=g).float()
        if kind == "equal":
            fill.zero_()
        if kind == "special":
            fill[::5], fill[1::5], fill[2::7], fill[3::7] = math.inf, -math.inf, math.nan, -0.0
        m.weight[p, :, s] = fill.double()
        m.dev["weight"][p.cuda(), :, s.cuda()] = fill.cuda()
    check_append(m, T, L - 50 if T == 40 else L, recent=2, w=w)


@pytest.mark.parametrize("T", [40, 64, 65, 3000])
@pytest.mark.parametrize("kind", ["spread", "coarse", "equal"])
def test_append_long_lists_with_ties(kind, T):
    """Lists long enough for several CTAs to share a head's candidates."""
    lens, H = [2500, 2311, -1], 2
    m = PagedMirror(lens, H, 64, 16, 2500)
    g = torch.Generator().manual_seed(T)
    w = torch.exp(torch.randn(3, H, T, generator=g))
    if kind != "spread":
        w = torch.randint(0, 3 if kind == "coarse" else 1, (3, H, T), generator=g).float()
        for n in range(2):
            p, s = m.where(n, lens[n])
            fill = torch.randint(0, 3 if kind == "coarse" else 1, (lens[n], H), generator=g).float()
            m.weight[p, :, s] = fill.double()
            m.dev["weight"][p.cuda(), :, s.cuda()] = fill.cuda()
    check_append(m, T, 2500, recent=20, sinks=3, w=w, counts=torch.tensor([T, T - 3, T], dtype=torch.int32))


def test_append_more_candidates_than_shared_memory_holds():
    N, H, T = 1, 1, 60000
    m = PagedMirror([0], H, 64, 64, 4096)
    w = torch.exp(torch.randn(N, H, T, generator=torch.Generator().manual_seed(2)))
    check_append(m, T, 4096, recent=16, sinks=4, w=w, fresh=True)
    m = PagedMirror([70000] * 160, H, 64, 64, 70000, spare=0)          # one CTA for each head's 70001 candidates
    m.append = lambda *a: None
    before = {k: m.dev[k].clone() for k in ("K", "pos")}
    cache = m.cache(ec)
    K = rand((160, H, 70, 64), BF, 3).cuda()
    w = torch.full((160, H, 70), 2.0, device="cuda")                   # above every cached weight: the lowest 70 rows leave
    order = [m.dev["weight"][m.dev["table"][n].long()].flatten()[:70000].argsort()[:70] for n in (0, 159)]
    ws = scratch(ec.ec_paged_append_workspace(cache, 70, 70000))
    ec.ec_paged_append(K, K, w, None, None, cache, False, 70000, 0, 0, ws)
    torch.cuda.synchronize()
    for n, low in zip((0, 159), order):
        rows = torch.sort(low)[0]
        page, slot = m.dev["table"][n].long()[rows // 64], rows % 64
        assert torch.equal(m.dev["K"][page, 0, slot].view(torch.int16), K[n, 0].view(torch.int16))
        changed = (m.dev["pos"] != before["pos"])[m.dev["table"][n].long()].flatten()[:70000]
        assert torch.equal(changed.nonzero()[:, 0], rows)
    assert m.dev["lens"].tolist() == [70000] * 160


@pytest.mark.parametrize("T", [0, 1, 30])
def test_append_shrinks_to_a_smaller_budget(T):
    m = PagedMirror([500, 64, 63, 10, 0], 2, 64, 16, 512)
    check_append(m, T, 64, recent=10, sinks=3, w=torch.rand(5, 2, T) if T else None)


@pytest.mark.parametrize("T,budget", [(640, 320), (1, 1), (7, 64), (1000, 1000), (5000, 100)])
def test_append_fresh_prompts(T, budget):
    N, H = 3, 2
    m = PagedMirror([17, 0, -1], H, 64, 16, budget if budget > 32 else 32)
    g = torch.Generator().manual_seed(T)
    w = torch.exp(2 * torch.randn(N, H, T, generator=g))
    w[w < 0.2] = 0.0
    counts = torch.tensor([T, max(1, T // 3), T], dtype=torch.int32)
    check_append(m, T, budget, recent=min(budget // 2, 16), sinks=min(budget // 4, 4), w=w, counts=counts, fresh=True)


def test_append_given_positions_decide_what_is_protected():
    N, H, T = 2, 2, 40
    m = PagedMirror([90, 50], H, 64, 16, 96)
    pos = torch.randint(0, 400, (N, H, T), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    check_append(m, T, 96, recent=20, sinks=30, w=torch.rand(N, H, T), pos=pos)


def test_append_does_not_follow_bad_pages():
    m = PagedMirror([40, 40], 1, 64, 16, 48)
    good = {k: v.clone() for k, v in m.dev.items()}
    m.dev["table"][1, 2] = 12345                                       # rows 32.. of problem 1
    cache = m.cache(ec)
    K = rand((2, 1, 4, 64), BF, 1).cuda()
    ws = scratch(ec.ec_paged_append_workspace(cache, 4, 48))
    ec.ec_paged_append(K, K, None, None, None, cache, False, 48, 4, 0, ws)
    torch.cuda.synchronize()
    assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE
    p = m.table[1].long()
    assert torch.equal(m.dev["K"][p].view(torch.int16), good["K"][p].view(torch.int16))   # nothing of problem 1 was written
    assert m.dev["lens"].tolist() == [44, 44]


# ---------------------------------------------------------------------------------------- whole steps

def run_steps(m, G, steps, budget, recent, sinks, use_graph=False, stream=None):
    N, H, D, dt = m.N, m.H, m.D, m.dtype
    scale, Hq = 1.0 / math.sqrt(D), H * G
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_step_workspace(cache, Hq, budget))
    q, k, v = (torch.empty(N, h, D, dtype=dt, device="cuda") for h in (Hq, H, H))
    out = torch.empty(N, Hq, D, dtype=dt, device="cuda")
    lse = torch.empty(N, Hq, device="cuda")
    ctx = torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream())

    def step():
        ec.ec_paged_decode_step(q, k, v, cache, scale, 1.0, budget, recent, sinks, out, lse, ws)
    torch.cuda.synchronize()
    graph = None
    with ctx:
        for i in range(steps):
            hq, hk, hv = rand((N, Hq, D), dt, 100 + i), rand((N, H, D), dt, 200 + i), rand((N, H, D), dt, 300 + i)
            for dst, src in ((q, hq), (k, hk), (v, hv)):
                dst.copy_(src)
            out.fill_(float("nan"))
            if use_graph:
                if graph is None:
                    torch.cuda.synchronize()
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        step()
                graph.replay()
            else:
                step()
            torch.cuda.current_stream().synchronize()
            ref, mass, dx = m.attention(hq, hk, hv, scale, True, 1.0)
            out_tol, lse_tol, w_tol = attention_bounds(ref, mass, dx, dt, G)
            m.append(hk[:, :, None], hv[:, :, None], ref[2][:, :, None], None, None, 1, False, budget, recent, sinks)
            assert ((out.cpu().double() - ref[0]).abs() <= out_tol).all(), f"step {i}"
            held = m.weight[torch.isfinite(m.weight)]
            m.assert_same_rows((i + 1) * (w_tol + float(held.max()) * 2.0 ** -22), f"step {i}")
    assert ec.ec_device_status(state_of(cache)) == ec.EC_OK


@pytest.mark.parametrize("G,dt,D", [(1, BF, 128), (4, HF, 64), (12, BF, 64)])
def test_steps_follow_the_definition(G, dt, D):
    run_steps(PagedMirror([40, 37, 0, -1, 12], 2, D, 16, 40, dt, G=G, ranked=True), G, 12, 40, 14, 2)


@pytest.mark.parametrize("page,rows", [(1, "tokens"), (1, "heads"), (5, "tokens"), (3, "heads")])
def test_steps_with_heads_side_by_side_in_memory(page, rows):
    """Weights and scores of several heads within 32 bytes, changed by different CTAs step after step."""
    run_steps(PagedMirror([70, 64, 70, 11], 8, 64, page, 70, rows=rows, G=2, ranked=True), 2, 8, 70, 12, 2)


@pytest.mark.parametrize("G", [2, 12])
@pytest.mark.parametrize("lens,budget", [([300, 150, 299, -1], 120), ([700], 650), ([2600, 2590], 2500)])
def test_steps_after_the_budget_shrank(lens, budget, G):
    """More rows leave than join: the first step brings every problem down to the new budget."""
    cap = max(lens) + 8
    run_steps(PagedMirror(lens, 2, 64, 16, cap, G=G, ranked=True, seed=budget), G, 2, budget, 14, 2)


def shift_off_16_bytes(t, by=1):
    held = torch.zeros(t.numel() + 4, dtype=t.dtype, device="cuda")
    moved = held[by:by + t.numel()].view(t.shape)
    moved.copy_(t)
    assert moved.data_ptr() % 16 == 4 * by
    return moved


@pytest.mark.parametrize("which", ["weight", "pos"])
@pytest.mark.parametrize("by", [1, 2])
def test_weights_and_positions_off_16_bytes(which, by):
    m = PagedMirror([100, 0, 1027], 3, 64, 16, 1100, G=2, ranked=True)
    m.dev[which] = shift_off_16_bytes(m.dev[which], by)
    check_attention(m, 2, accumulate=True)
    m = PagedMirror([64, 62, 9], 3, 64, 16, 64, G=2, ranked=True)
    m.dev[which] = shift_off_16_bytes(m.dev[which], by)
    run_steps(m, 2, 6, 64, 8, 1)


@pytest.mark.parametrize("page", [4, 12, 20])
@pytest.mark.parametrize("length", [1, 2, 3, 4, 5, 511, 514])
def test_steps_at_every_rest_of_four_rows(length, page):
    run_steps(PagedMirror([length, max(0, length - 2)], 2, 64, page, 520, G=3, ranked=True), 3, 6, length + 3, 2, 1)


def test_steps_of_long_problems():
    """Rows beyond what one CTA brings up to date by itself."""
    run_steps(PagedMirror([5000, 4700], 2, 64, 64, 5000, G=1, ranked=True), 1, 3, 5000, 14, 2)


def test_steps_of_many_units():
    lens = [60 - (n % 9) for n in range(40)]
    lens[3], lens[17] = -1, 0
    run_steps(PagedMirror(lens, 16, 64, 16, 60, G=1, ranked=True), 1, 2, 60, 8, 2)


def test_steps_captured_once_and_replayed():
    run_steps(PagedMirror([100, 97, -1], 2, 64, 16, 100, ranked=True, G=2), 2, 8, 100, 10, 1, use_graph=True)


def test_steps_on_another_stream():
    run_steps(PagedMirror([64, 20], 2, 64, 32, 64, ranked=True), 1, 4, 64, 8, 0, stream=torch.cuda.Stream())


def test_two_caches_share_a_workspace_in_one_stream():
    """Two captured steps of different caches over one workspace, replayed in turn, give what separate ones give."""
    outs = []
    for shared in (True, False):
        ms = [PagedMirror([50, 33], 2, 64, 16, 64, seed=s) for s in (1, 2)]
        caches = [m.cache(ec) for m in ms]
        need = ec.ec_paged_step_workspace(caches[0], 4, 64)
        one = scratch(need)
        graphs, got = [], []
        for i, c in enumerate(caches):
            q, k, v = rand((2, 4, 64), BF, i).cuda(), rand((2, 2, 64), BF, 5 + i).cuda(), rand((2, 2, 64), BF, 7 + i).cuda()
            out = torch.zeros(2, 4, 64, dtype=BF, device="cuda")
            ws = one if shared else scratch(need)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                ec.ec_paged_decode_step(q, k, v, c, 0.125, 1.0, 64, 4, 0, out, None, ws)
            graphs.append((g, q, k, v, ws))
            got.append(out)
        for _ in range(20):
            for g, *_rest in graphs:
                g.replay()
        torch.cuda.synchronize()
        outs.append([o.clone() for o in got] + [m.dev[x].clone() for m in ms for x in ("K", "weight", "pos", "lens")])
    for a, b in zip(*outs):
        assert torch.equal(a.nan_to_num(7.0) if a.is_floating_point() else a, b.nan_to_num(7.0) if b.is_floating_point() else b)


def test_two_caches_on_two_streams_at_once():
    """Each with its own description and workspace, interleaved without waiting; the same as one after the other."""
    def build():
        ms = [PagedMirror([700, 400, 33, -1], 4, 128, 16, 704, seed=s, ranked=True, G=2) for s in (3, 4)]
        ins = [[rand((4, h, 128), BF, 20 * s + h).cuda() for h in (8, 4, 4)] for s in (0, 1)]
        cs = [m.cache(ec) for m in ms]
        ws = [scratch(ec.ec_paged_step_workspace(c, 8, 704)) for c in cs]
        outs = [torch.zeros(30, 4, 8, 128, dtype=BF, device="cuda") for _ in cs]
        return ms, ins, cs, ws, outs
    got = []
    for at_once in (True, False):
        ms, ins, cs, ws, outs = build()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if at_once else [torch.cuda.current_stream()] * 2
        torch.cuda.synchronize()
        for i in range(30):
            for (q, k, v), c, w, o, st in zip(ins, cs, ws, outs, streams):
                with torch.cuda.stream(st):
                    ec.ec_paged_decode_step(q, k, v, c, 0.088, 1.0, 704, 16, 2, o[i], None, w)
        torch.cuda.synchronize()
        got.append(outs + [m.dev[x] for m in ms for x in ("pos", "lens", "seen")] + [m.dev["weight"].nan_to_num(7.0) for m in ms])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_shared_pages_can_be_read():
    """A common beginning in the same pages for two problems."""
    m = PagedMirror([96, 80], 2, 64, 32, 96)
    for t in (m.table, m.dev["table"]):
        t[1, :2] = t[0, :2]
    check_attention(m, 3)


def test_values_that_are_infinite_stay_where_they_belong():
    m = PagedMirror([100, 60], 1, 64, 16, 112)
    p, s = m.where(0, 100)
    for pool in (m.V, m.dev["V"]):
        pool[p[7], 0, s[7], 5] = math.inf                              # one dimension of one row
    cache = m.cache(ec)
    q, k, v = (rand((2, 1, 64), BF, i).cuda() for i in range(3))
    out = torch.empty_like(q)
    ws = scratch(ec.ec_paged_attention_workspace(cache, 1, False))
    ec.ec_paged_attention(q, k, v, cache, 0.125, False, 1.0, out, None, None, ws)
    torch.cuda.synchronize()
    fine = torch.isfinite(out)
    assert not fine[0, 0, 5] and int((~fine).sum()) == 1


def test_offsets_past_32_bits():
    """Rows more than 2^32 bytes and 2^31 elements into the pool."""
    H, D, page, n_pages = 4, 128, 128, 36000                           # 36000 * 4 * 128 * 128 elements = 4.7 GB a pool
    K = torch.empty((n_pages, H, page, D), dtype=BF, device="cuda")
    V = torch.empty_like(K)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32)
    m = PagedMirror([300], H, D, page, 384)
    for pool, small in ((K, m.dev["K"]), (V, m.dev["V"])):
        pool[table[0].long().cuda()] = small[m.table[0].long().cuda()]
    weight = torch.zeros((n_pages, H, page), device="cuda")
    pos = torch.zeros((n_pages, H, page), dtype=torch.int32, device="cuda")
    state = torch.empty(ec.ec_paged_state_bytes(1), dtype=torch.uint8, device="cuda")
    big = ec.ec_paged_init(K, V, weight, pos, table.cuda(), m.dev["lens"], m.dev["seen"], state)
    small = m.cache(ec)
    q = rand((1, 8, D), BF, 1).cuda()
    outs = []
    for c in (small, big):
        out = torch.empty_like(q)
        ws = scratch(ec.ec_paged_attention_workspace(c, 8, False))
        ec.ec_paged_attention(q, None, None, c, 0.1, False, 1.0, out, None, None, ws)
        outs.append(out.clone())
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    one = rand((1, H, 1, D), BF, 4).cuda()
    ws = scratch(ec.ec_paged_append_workspace(big, 1, 384))
    ec.ec_paged_append(one, one, None, None, None, big, False, 384, 1, 0, ws)
    torch.cuda.synchronize()
    assert torch.equal(K[n_pages - 2, :, 300 - 256], one[0, :, 0]) and int(m.dev["lens"][0]) == 301
    assert ec.ec_device_status(state) == ec.EC_OK


# ---------------------------------------------------------------------------------------- as they are used

def adopt(session):
    """A host mirror of a session's cache as it is now."""
    s = session
    m = PagedMirror([0] * s.N, s.H, s.D, s.Kp.shape[2], s.budget, s.Kp.dtype, device=None, spare=0)
    m.table, m.lens, m.seen = s.table.cpu(), s.lens.cpu().clone(), s.seen.cpu().clone()
    m.K, m.V, m.weight, m.pos = s.Kp.cpu().clone(), s.Vp.cpu().clone(), s.weight.cpu().double(), s.pos.cpu().clone()
    m.dev = dict(K=s.Kp, V=s.Vp, weight=s.weight, pos=s.pos, lens=s.lens, seen=s.seen)
    return m


@pytest.mark.parametrize("with_output", [False, True])
def test_prompt_then_steps_then_a_new_prompt(with_output):
    N, H, D, T, budget = 3, 2, 64, 150, 80
    s = PagedCacheSession(N, H, D, budget, recent=12, sinks=2, scale=0.125, page_size=32)
    s.lens[1] = -1                                                     # an empty place
    for round_ in range(2):
        Q, K, V = (rand((N, H, T, D), BF, 10 * round_ + i) for i in range(3))
        m = adopt(s)
        out = torch.empty(N, H, T, D, dtype=BF, device="cuda") if with_output else None
        scores = torch.empty(N, H, T, device="cuda")
        s.prompt(Q.cuda(), K.cuda(), V.cuda(), out, scores=scores)
        torch.cuda.synchronize()
        scores = scores.cpu()
        x = torch.einsum("nhmd,nhkd->nhmk", Q.double(), K.double()) * 0.125
        p = torch.softmax(x.masked_fill(torch.ones(T, T).triu(1).bool(), -math.inf), -1)
        assert (scores.double() - p.sum(2)).abs().max() <= 1e-3 * p.sum(2).max()
        if with_output:
            assert ((out.cpu().double() - p @ V.double()).abs() <= 2e-2 + 2.0 ** -8 * (p @ V.double()).abs()).all()
        m.append(K, V, scores, None, None, T, True, budget, 12, 2)
        m.assert_same_rows(0.0, "prompt")
        for i in range(10):
            q, k, v = (rand((N, H, D), BF, 100 + 3 * i + j) for j in range(3))
            got = torch.empty(N, H, D, dtype=BF, device="cuda")
            s.decode(q.cuda(), k.cuda(), v.cuda(), got)
            ref, mass, dx = m.attention(q, k, v, 0.125, True)
            out_tol, _, w_tol = attention_bounds(ref, mass, dx, BF, 1)
            m.append(k[:, :, None], v[:, :, None], ref[2][:, :, None], None, None, 1, False, budget, 12, 2)
            assert ((got.cpu().double() - ref[0]).abs() <= out_tol).all()
            m.assert_same_rows((i + 1) * (w_tol + float(m.weight.max()) * 2.0 ** -22), f"step {i}")
        assert s.status() == ec.EC_OK and s.lens.tolist() == [budget, -1, budget] and s.seen.tolist()[0] == T + 10


def test_a_compacted_cache_in_pages_answers_as_the_dense_one():
    """Merged rows of ec_select_merge, taken into pages with the anchors' scores and positions."""
    N, H, D, T, keep = 2, 4, 128, 200, 100
    Q, K, V = (rand((N, H, T, D), BF, i).cuda() for i in range(3))
    scores = torch.empty(N, H, T, device="cuda")
    ws = scratch(max(ec.ec_importance_workspace(N, H, T, D), ec.ec_select_merge_workspace(N, H, T, D, keep, ec.EC_PER_HEAD)))
    ec.ec_importance(Q, K, scores, None, 0.088, ws)
    Kc, Vc = (torch.empty(N, H, keep, D, dtype=BF, device="cuda") for _ in range(2))
    anchors = torch.empty(N, H, keep, dtype=torch.int32, device="cuda")
    ec.ec_select_merge(K, V, scores, keep, ec.EC_PER_HEAD, True, Kc, Vc, anchors, None, ws)
    s = PagedCacheSession(N, H, D, keep, recent=8, sinks=1, scale=0.088, page_size=16)
    app = scratch(ec.ec_paged_append_workspace(s.cache, keep, keep))
    ec.ec_paged_append(Kc, Vc, scores.gather(2, anchors.long()), anchors, None, s.cache, True, keep, 8, 1, app)
    s.seen.fill_(T)                                                    # the rows stand for T tokens
    dense = ec.ec_cache_init(Kc, Vc, keep, keep, 16)
    wd = scratch(ec.ec_decode_workspace(dense))
    q, k, v = (rand((N, H, D), BF, 7 + i).cuda() for i in range(3))
    a, b = torch.empty_like(q), torch.empty_like(q)
    s.decode(q, k, v, a)
    ec.ec_decode_step(q, k, v, dense, 0.088, b, wd)
    torch.cuda.synchronize()
    # both round the result once; the dense kernel and this one each carry fp32 sums besides
    tol = torch.finfo(BF).eps * b.float().abs() + 2.0 ** -12
    assert ((a.float() - b.float()).abs() <= tol).all()
    new = (s.pos == T).nonzero()
    assert new.shape[0] == N * H and s.lens.tolist() == [keep] * N and s.seen.tolist() == [T + 1] * N


def test_a_captured_prompt_keeps_its_workspaces():
    """Prompts of other lengths between the replays of a captured one change nothing of it."""
    N, H, D, T = 2, 2, 64, 200
    s = PagedCacheSession(N, H, D, 96, recent=8, sinks=2, scale=0.125, page_size=32)
    Q, K, V = (rand((N, H, T, D), BF, i).cuda() for i in range(3))
    s.prompt(Q, K, V)
    kept = lambda: [t.clone() for t in (s.weight, s.pos, s.lens, s.seen)]  # noqa: E731
    want = kept()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.prompt(Q, K, V)
    held = []
    for other in (70, 333):
        x = [rand((N, H, other, D), BF, other + i).cuda() for i in range(3)]
        s.prompt(*x)
        held.append([torch.full((1 << 16,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(20)])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept(), want):
            assert torch.equal(a, b)
        assert all(bool((t == 0x5A).all()) for t in held[-1])


def test_a_prompt_of_other_sizes_is_refused():
    s = PagedCacheSession(2, 2, 64, 64, 4, 0, 0.125)
    x = torch.zeros(2, 2, 70, 64, dtype=BF, device="cuda")
    good = dict(Q=x, K=x, V=x, out=torch.empty_like(x), lse=torch.empty(2, 2, 70, device="cuda"))
    wide = torch.zeros(4, 2, 70, 64, dtype=BF, device="cuda")
    for name, bad in (("Q", wide), ("K", wide), ("V", wide), ("Q", x[:, :, :69]), ("K", x.half()), ("out", x[:1]), ("Q", x.cpu()),
                      ("lse", torch.empty(2, 2, 69, device="cuda")), ("K", x[0])):
        with pytest.raises(ValueError):
            s.prompt(**{**good, name: bad})
    with pytest.raises(ValueError):
        s.prompt(wide, wide, wide)
    with pytest.raises(ValueError):
        s.prompt(**good, scores=torch.empty(2, 2, 71, device="cuda"))
    assert s.lens.tolist() == [0, 0]
    s.prompt(**good)
    assert s.lens.tolist() == [64, 64]


def test_binding_refuses_wrong_tensors():
    s = PagedCacheSession(2, 2, 64, 64, 4, 0, 0.125)
    q = torch.zeros(2, 2, 64, dtype=BF, device="cuda")
    out = torch.empty_like(q)
    for bad in (q.half(), q[:1], q.cpu(), torch.zeros(2, 64, 2, dtype=BF, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            s.decode(q, bad, q, out)
    with pytest.raises(ValueError):
        ec.ec_paged_init(s.Kp, s.Vp.transpose(1, 2), s.weight, s.pos, s.table, s.lens, s.seen, s.state)
    with pytest.raises(ValueError):
        ec.ec_paged_init(s.Kp, s.Vp, s.weight[:1], s.pos, s.table, s.lens, s.seen, s.state)
    with pytest.raises(ValueError):
        ec.ec_paged_init(s.Kp, s.Vp, s.weight, s.pos, s.table, s.lens, s.seen, s.state[:256])
    with pytest.raises(ec.EcError) as e:
        ec.ec_paged_append(q[:, :, None], q[:, :, None], None, None, None, s.cache, False, 65, 4, 0, s.ws_step)
    assert e.value.status == ec.EC_ERR_ARG
    with pytest.raises(ec.EcError) as e:
        ec.ec_paged_decode_step(q, q, q, s.cache, 0.125, 1.0, 64, 4, 0, out, None, s.ws_step[:256])
    assert e.value.status == ec.EC_ERR_WORKSPACE
    assert s.lens.tolist() == [0, 0]
    half = PagedCacheSession(2, 2, 64, 64, 4, 0, 0.125, dtype=HF)
    x = torch.zeros(2, 2, 70, 64, dtype=HF, device="cuda")
    with pytest.raises(ValueError):
        half.prompt(x, x, x)
    with pytest.raises(ValueError):
        PagedCacheSession(2, 2, 64, 64, 4, 0, 0.125, Hq=4).prompt(x.bfloat16(), x.bfloat16(), x.bfloat16())
