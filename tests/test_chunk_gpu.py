"""A chunk of new tokens on a paged cache, on the GPU, against plain 64-bit forms: attention and gathered weights."""
import math

import pytest
import torch

from chunk_reference import ChunkExact
from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from test_paged_gpu import BF, HF, rand, scratch, state_of

pytestmark = pytest.mark.gpu


def pack(counts, gap=0):
    """starts of packed problems, `gap` tokens of nobody in front of each; tokens in all, with as many behind the last."""
    starts, at = [], 0
    for c in counts:
        at += gap
        starts.append(at)
        at += max(c, 0)
    return torch.tensor(starts, dtype=torch.int32), at + gap


def mirror(lens, H, D, page, dt=BF, rows="heads", seed=0, cap=None, garbage=float("nan")):
    return PagedMirror(lens, H, D, page, cap or max(max(lens), 1), dt, rows, seed, garbage=garbage)


def check(m, counts, G, scale=None, decay=0.9, q=None, gap=0, seed=5, drop=(), status=ec.EC_OK, twice=True, weights=True, what=""):
    """Runs both calls, compares them with the definition, and what must not change with what was there."""
    H, D, dt = m.H, m.D, m.dtype
    scale = scale or 1.0 / math.sqrt(D)
    starts, tokens = pack(counts, gap)
    counts = torch.tensor(counts, dtype=torch.int32)
    q = rand((tokens, H * G, D), dt, seed) if q is None else q
    cache = m.cache(ec)
    before = m.dev["weight"].clone()
    m.weight = before.cpu().double()
    ref = ChunkExact(m, q, starts, counts, scale, drop=drop)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, H * G))
    out = torch.full((tokens, H * G, D), 7.0, dtype=dt, device="cuda")
    lse = torch.full((tokens, H * G), 7.0, device="cuda")
    qd, sd, cd = q.cuda(), starts.cuda(), counts.cuda()
    first = None
    for _ in range(2 if twice else 1):
        ec.ec_paged_chunk_attention(qd, sd, cd, cache, scale, out, lse, ws)
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        if first:
            assert all(torch.equal(a.nan_to_num(77.0), b.nan_to_num(77.0)) for a, b in zip(first, got)), what + ": two runs differ"
        first = got
    assert ec.ec_device_status(state_of(cache)) == status
    ref.assert_out(out, lse, what)
    nobody = ~ref.owned
    assert (out.cpu()[nobody] == 7.0).all() and (lse.cpu()[nobody] == 7.0).all(), what + ": rows of nobody"
    m.assert_same_rows(0.0, what)
    if not weights:
        return ref, out, lse
    z = ref.lse.float().cuda()
    ref_w = ChunkExact(m, q, starts, counts, scale, decay, lse=ref.lse.float(), drop=drop)
    first = None
    for _ in range(2 if twice else 1):
        m.dev["weight"].copy_(before)
        ec.ec_paged_chunk_weights(qd, z, sd, cd, cache, scale, decay, ws)
        torch.cuda.synchronize()
        got = m.dev["weight"].clone()
        assert first is None or torch.equal(first.nan_to_num(77.0), got.nan_to_num(77.0)), what + ": two runs of the weights differ"
        first = got
    ref_w.assert_weights(m.dev["weight"], what)
    assert ec.ec_device_status(state_of(cache)) == status
    return ref, out, lse


EDGE = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 200]
BEFORE = [0, 1, 15, 96, 0, 17, 64, 63, 1, 128, 300, 40, 129]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("G", [1, 3, 4, 7, 16])
def test_edges_of_chunk_and_length(G, dt, D):
    counts = [max(1, c // G) if c else 0 for c in EDGE]
    check(mirror([b + c for b, c in zip(BEFORE, counts)], 2, D, 16, dt), counts, G, gap=3)


@pytest.mark.parametrize("tokens", [127, 128, 129, 255, 256, 257, 511])
def test_one_head_around_the_tiles(tokens):
    check(mirror([tokens + 5], 1, 128, 64), [tokens], 1)


@pytest.mark.parametrize("G,counts", [(33, [5, 9]), (64, [3, 2]), (100, [1, 4]), (128, [3, 1])])
def test_wide_groups(G, counts):
    check(mirror([c + 70 for c in counts], 2, 64, 16), counts, G)


@pytest.mark.parametrize("rows", ["heads", "tokens"])
@pytest.mark.parametrize("page", [1, 2, 3, 4, 5, 8, 12, 16, 24, 48, 64, 96, 100, 128, 192, 256])
def test_pages_of_all_sizes(page, rows):
    check(mirror([150, 1, 333, 64], 2, 64, page, rows=rows, cap=340), [20, 1, 70, 64], 2)


def test_few_tokens_on_long_sequences_are_spread_over_the_gpu():
    check(mirror([20011, 3, 7000], 2, 128, 64), [3, 1, 8], 4)


def test_many_units_and_whole_prompts():
    check(mirror([300 + 7 * i for i in range(40)], 3, 64, 16), [1 + 5 * i for i in range(40)], 2)


def test_a_long_prompt():
    check(mirror([2100], 2, 128, 128), [2100], 2, decay=0.999)


@pytest.mark.parametrize("decay", [1.0, 0.5, 1e-6])
def test_decay(decay):
    check(mirror([90, 300], 2, 64, 16), [40, 130], 2, decay=decay)


def test_empty_places_and_counts_past_the_length():
    """A problem without rows, an empty place with tokens, and more tokens than rows: the first of them see nothing."""
    m = mirror([0, 30, 5, 200], 2, 64, 16)
    m.lens[0] = -1
    m.dev["lens"][0] = -1
    ref, out, lse = check(m, [4, 0, 9, 201], 3, gap=2)
    assert (out.cpu()[2:6] == 0).all() and torch.isinf(lse.cpu()[2:6]).all()
    assert torch.isinf(ref.lse).any()


def test_nothing_at_all():
    m = mirror([30, 5], 2, 64, 16)
    check(m, [0, 0], 2, gap=4)
    m.dev["lens"].fill_(-1)
    m.lens.fill_(-1)
    check(m, [0, -3], 2, gap=4)


def test_packed_rows_by_strides():
    """Queries out of a projection's output, results into the middle of something wider, heads in front of tokens."""
    m = mirror([77, 40], 2, 64, 16)
    starts, tokens = pack([50, 33])
    G, D = 2, 64
    q = rand((tokens, 4, D), BF, 3)
    wide = torch.randn(tokens, 4 + 4, D + 64, dtype=BF, device="cuda")
    wide[:, 2:6, 64:] = q.cuda()
    by_head = torch.full((4 + 2, tokens, D), 7.0, dtype=BF, device="cuda")
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 4))
    counts = torch.tensor([50, 33], dtype=torch.int32)
    lse = torch.empty(tokens, 4, device="cuda")
    view = by_head[1:5].transpose(0, 1)
    ec.ec_paged_chunk_attention(wide[:, 2:6, 64:], starts.cuda(), counts.cuda(), cache, 0.125, view, lse, ws)
    ref = ChunkExact(m, q, starts, counts, 0.125)
    ref.assert_out(view, lse)
    assert (by_head[0] == 7.0).all() and (by_head[5] == 7.0).all()
    ec.ec_paged_chunk_weights(wide[:, 2:6, 64:], ref.lse.float().cuda(), starts.cuda(), counts.cuda(), cache, 0.125, 0.9, ws)
    ChunkExact(m, q, starts, counts, 0.125, 0.9, lse=ref.lse.float()).assert_weights(m.dev["weight"])


@pytest.mark.parametrize("page", [4, 16, 64])
def test_bad_pages_are_not_followed(page):
    m = mirror([200, 90, 130], 2, 64, page, cap=208)
    drop = set()
    for n, p, bad in ((0, 1, -1), (0, 2, 1 << 20), (2, 0, -5)):
        m.dev["table"][n, p] = bad
        drop |= {(n, j) for j in range(p * page, (p + 1) * page)}
    check(m, [30, 90, 7], 2, drop=drop, status=ec.EC_ERR_PAGE)


def test_starts_and_lengths_out_of_range():
    m = mirror([50, 50, 50], 2, 64, 16)
    q = rand((60, 2, 64), BF, 1).cuda()
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 2))
    for starts, counts in (([0, 55, 20], [20, 6, 20]), ([0, -1, 20], [20, 2, 20]), ([0, 1 << 30, 20], [20, 1, 20])):
        out, lse = torch.full_like(q, 7.0), torch.full((60, 2), 7.0, device="cuda")
        s, c = torch.tensor(starts, dtype=torch.int32), torch.tensor(counts, dtype=torch.int32)
        ec.ec_paged_chunk_attention(q, s.cuda(), c.cuda(), cache, 0.125, out, lse, ws)
        assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE
        ref = ChunkExact(m, q.cpu(), s, torch.tensor([20, 0, 20]), 0.125)
        ref.assert_out(out, lse)
        assert (out.cpu()[~ref.owned] == 7.0).all()
        cache = m.cache(ec)
    # a length past the table is cut
    m.dev["lens"][1] = 5000
    out, lse = torch.empty_like(q), torch.empty(60, 2, device="cuda")
    s, c = torch.tensor([0, 20, 40], dtype=torch.int32).cuda(), torch.tensor([20, 20, 20], dtype=torch.int32).cuda()
    ec.ec_paged_chunk_attention(q, s, c, cache, 0.125, out, lse, ws)
    assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE


# ------------------------------------------------------------------ values

@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_reach_only_those_who_see_them(dt, bad):
    """A value row of one new token: tokens in front of it must not notice."""
    m = mirror([170, 140, 60], 2, 64, 16, dt)
    for n, row in ((0, 150), (1, 139), (2, 0)):
        p, s = int(m.table[n][row // 16]), row % 16
        for where in (m.V, m.dev["V"]):
            where[p, 1, s, 5] = bad
    counts, G = [60, 140, 60], 2
    starts, tokens = pack(counts)
    q = rand((tokens, 4, 64), dt, 8)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 4))
    out = torch.empty(tokens, 4, 64, dtype=dt, device="cuda")
    ec.ec_paged_chunk_attention(q.cuda(), starts.cuda(), torch.tensor(counts, dtype=torch.int32).cuda(), cache, 0.125, out, None, ws)
    ref = ChunkExact(m, q, starts, torch.tensor(counts), 0.125)
    got = out.cpu().double()
    seen = torch.isnan(ref.out)
    assert seen.any() and not seen.all()
    assert not torch.isfinite(got[seen]).any()
    assert ((got - ref.out).abs()[~seen] <= ref.out_tol[~seen]).all()


def test_a_key_or_query_that_is_not_a_number_stays_where_it_belongs():
    m = mirror([150, 150], 1, 64, 16)
    p, s = int(m.table[0][140 // 16]), 140 % 16
    for where in (m.K, m.dev["K"]):
        where[p, 0, s] = float("nan")
    q = rand((300, 1, 64), BF, 2)
    q[200] = float("nan")
    starts, counts = torch.tensor([0, 150], dtype=torch.int32), torch.tensor([150, 150], dtype=torch.int32)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 1))
    out, lse = torch.empty(300, 1, 64, dtype=BF, device="cuda"), torch.empty(300, 1, device="cuda")
    ec.ec_paged_chunk_attention(q.cuda(), starts.cuda(), counts.cuda(), cache, 0.125, out, lse, ws)
    bad = torch.zeros(300, dtype=torch.bool)
    bad[140:150] = True
    bad[200] = True
    assert torch.equal(torch.isnan(out.cpu()).all(-1)[:, 0], bad) and torch.equal(torch.isnan(lse.cpu())[:, 0], bad)
    assert torch.isfinite(out.cpu()[~bad]).all()


@pytest.mark.parametrize("token", [0, 1, 2, 8, 77, 255])
def test_a_query_that_is_not_a_number_reaches_every_row_that_it_sees(token):
    """Its normaliser is not a number, and so is the weight of each row that it sees; the others keep theirs."""
    length, count = 700, 256
    m = mirror([length, 90], 1, 64, 16)
    q = rand((count + 90, 1, 64), BF, 2)
    q[token] = float("nan")
    starts, counts = torch.tensor([0, count], dtype=torch.int32), torch.tensor([count, 90], dtype=torch.int32)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 1))
    out, lse = torch.empty(count + 90, 1, 64, dtype=BF, device="cuda"), torch.empty(count + 90, 1, device="cuda")
    ec.ec_paged_chunk_attention(q.cuda(), starts.cuda(), counts.cuda(), cache, 0.125, out, lse, ws)
    ec.ec_paged_chunk_weights(q.cuda(), lse, starts.cuda(), counts.cuda(), cache, 0.125, 1.0, ws)
    weight = m.dev["weight"].cpu()
    for n, rows in ((0, length), (1, 90)):
        page, slot = m.where(n, rows)
        bad = torch.isnan(weight[page, 0, slot])
        sees = torch.arange(rows) <= length - count + token if n == 0 else torch.zeros(rows, dtype=torch.bool)
        assert torch.equal(bad, sees)


@pytest.mark.parametrize("dt", [BF, HF])
def test_scores_of_minus_infinity(dt):
    """Keys that give -inf: rows that nothing is left of are zero, the others do without them."""
    m = mirror([40, 200], 1, 64, 16, dt)
    inf = float("inf")
    q = rand((60, 1, 64), dt, 4).abs() + 0.5
    for n, rows in ((0, range(40)), (1, range(0, 200, 3))):
        for j in rows:
            p, s = int(m.table[n][j // 16]), j % 16
            for where in (m.K, m.dev["K"]):
                where[p, 0, s] = 0.0
                where[p, 0, s, 0] = -inf
    ref, out, lse = check(m, [20, 40], 1, q=q)
    assert (out.cpu()[:20] == 0).all() and torch.isinf(lse.cpu()[:20]).all()


@pytest.mark.parametrize("dt,top", [(BF, 1e18), (HF, 6e4)])
def test_scores_as_large_as_the_type_allows(dt, top):
    """One key leads by far: its value comes out, whatever the size of the scores."""
    m = mirror([130, 300], 1, 64, 16, dt)
    q = torch.zeros(60, 1, 64, dtype=dt)
    q[:, 0, 0] = top
    for n, length in enumerate((130, 300)):
        for j in range(length):
            p, s = int(m.table[n][j // 16]), j % 16
            for where in (m.K, m.dev["K"]):
                where[p, 0, s, 0] = top if j == 7 else -top * (j % 5) / 5
    starts, counts = torch.tensor([0, 20], dtype=torch.int32), torch.tensor([20, 40], dtype=torch.int32)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 1))
    out, lse = torch.empty(60, 1, 64, dtype=dt, device="cuda"), torch.empty(60, 1, device="cuda")
    ec.ec_paged_chunk_attention(q.cuda(), starts.cuda(), counts.cuda(), cache, 1.0, out, lse, ws)
    for n, sl in ((0, slice(0, 20)), (1, slice(20, 60))):
        p, s = int(m.table[n][0]), 7
        want = m.V[p, 0, s]
        assert torch.equal(out[sl, 0].cpu(), want[None].expand_as(out[sl, 0].cpu()))
    assert torch.isfinite(lse).all() and (lse > 0).all()


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("scale", [1e-30, 1e-4, 3.0])
def test_scales(dt, scale):
    check(mirror([130, 300], 2, 64, 16, dt), [33, 150], 2, scale=scale)


@pytest.mark.parametrize("dt", [BF, HF])
def test_rows_far_below_a_leading_one_count(dt):
    """A row that leads by 17.5 nats with a value of zero: the output is made of the others."""
    m = mirror([300], 1, 64, 16, dt)
    q = torch.zeros(40, 1, 64, dtype=dt)
    q[:, 0, 0] = 1.0
    for where in (m.K, m.dev["K"]):
        where[:, :, :, :] = torch.nan_to_num(where, nan=0.0)
        where[:, :, :, 0] = 0.0
    p, s = int(m.table[0][9 // 16]), 9 % 16
    for where in (m.K, m.dev["K"]):
        where[p, 0, s, 0] = 17.5
    for where in (m.V, m.dev["V"]):
        where[p, 0, s] = 0.0
    check(m, [40], 1, q=q, scale=1.0)


# ------------------------------------------------------------------ how it is called

def test_one_token_gathers_what_the_single_call_gathers():
    lens, G = [130, 7, 64], 4
    a, b = (mirror(lens, 2, 64, 16, seed=3) for _ in range(2))
    q = rand((3, 2 * G, 64), BF, 1).cuda()
    ones, starts = torch.ones(3, dtype=torch.int32, device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda")
    ca, cb = a.cache(ec), b.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(ca, 2 * G))
    out, lse = torch.empty_like(q), torch.empty(3, 2 * G, device="cuda")
    ec.ec_paged_chunk_attention(q, starts, ones, ca, 0.125, out, lse, ws)
    ec.ec_paged_chunk_weights(q, lse, starts, ones, ca, 0.125, 0.75, ws)
    ws2 = scratch(ec.ec_paged_attention_workspace(cb, 2 * G, True))
    out2, lse2 = torch.empty_like(q), torch.empty(3, 2 * G, device="cuda")
    ec.ec_paged_attention(q, None, None, cb, 0.125, True, 0.75, out2, lse2, None, ws2)
    assert torch.allclose(lse, lse2, rtol=0, atol=2e-5)
    assert torch.allclose(a.dev["weight"].nan_to_num(0), b.dev["weight"].nan_to_num(0), rtol=3e-5, atol=3e-5)
    assert (out.float() - out2.float()).abs().max() <= 0.02


def test_a_captured_call_replayed_on_other_lengths():
    m = mirror([250, 250, 250], 2, 64, 16)
    G, tokens = 2, 300
    q = rand((tokens, 4, 64), BF, 6)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 4))
    qd = q.cuda()
    out, lse = torch.full((tokens, 4, 64), 7.0, dtype=BF, device="cuda"), torch.empty(tokens, 4, device="cuda")
    starts, counts = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ec.ec_paged_chunk_attention(qd, starts, counts, cache, 0.125, out, lse, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            ec.ec_paged_chunk_attention(qd, starts, counts, cache, 0.125, out, lse, ws)
            ec.ec_paged_chunk_weights(qd, lse, starts, counts, cache, 0.125, 0.9, ws)
    torch.cuda.synchronize()
    for c, lens in (([10, 100, 1], [250, 130, 4]), ([200, 0, 90], [200, 17, 90]), ([1, 1, 1], [1, 250, 100])):
        s, _ = pack(c)
        starts.copy_(s)
        counts.copy_(torch.tensor(c, dtype=torch.int32))
        m.lens = torch.tensor(lens, dtype=torch.int32)
        m.dev["lens"].copy_(m.lens)
        m.weight = m.dev["weight"].cpu().double()
        g.replay()
        torch.cuda.synchronize()
        ref = ChunkExact(m, q, s, torch.tensor(c), 0.125, 0.9)
        ref.assert_out(out, lse)
        ChunkExact(m, q, s, torch.tensor(c), 0.125, 0.9, lse=lse.cpu()).assert_weights(m.dev["weight"])


def test_two_caches_on_two_streams_at_once():
    jobs = []
    for i in range(2):
        m = mirror([900, 40, 300], 2, 64, 16, seed=i)
        starts, tokens = pack([60, 40, 1])
        q = rand((tokens, 4, 64), BF, 20 + i)
        cache = m.cache(ec)
        jobs.append((m, q, q.cuda(), starts, starts.cuda(), cache, scratch(ec.ec_paged_chunk_workspace(cache, 4)),
                     torch.empty(tokens, 4, 64, dtype=BF, device="cuda"), torch.empty(tokens, 4, device="cuda"), torch.cuda.Stream()))
    counts = torch.tensor([60, 40, 1], dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    for _ in range(20):
        for m, q, qd, s, sd, cache, ws, out, lse, st in jobs:
            with torch.cuda.stream(st):
                ec.ec_paged_chunk_attention(qd, sd, counts, cache, 0.125, out, lse, ws)
    torch.cuda.synchronize()
    for m, q, qd, s, sd, cache, ws, out, lse, st in jobs:
        ChunkExact(m, q, s, counts.cpu(), 0.125).assert_out(out, lse)


def test_problems_that_share_pages():
    """Two problems on one prefix: pages are read by both."""
    m = mirror([200, 200], 2, 64, 16)
    m.table[1, :10] = m.table[0, :10]
    m.dev["table"].copy_(m.table)
    check(m, [40, 40], 2, weights=False)


def test_no_normaliser_wanted():
    m = mirror([100], 2, 64, 16)
    q = rand((30, 2, 64), BF, 1)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 2))
    out = torch.empty(30, 2, 64, dtype=BF, device="cuda")
    z = torch.zeros(1, dtype=torch.int32)
    ec.ec_paged_chunk_attention(q.cuda(), z.cuda(), torch.tensor([30], dtype=torch.int32).cuda(), cache, 0.125, out, None, ws)
    ChunkExact(m, q, z, torch.tensor([30]), 0.125).assert_out(out)


def test_offsets_past_32_bits():
    """Pages more than 4 GiB apart, in K and in V."""
    n_pages, H, page, D = 3, 1, 16, 64
    step = (5 << 30) // 2 // 2                                 # elements between pages: 2.5 GiB
    big = torch.empty(2 * step + H * page * D, dtype=BF, device="cuda")
    big2 = torch.empty_like(big)
    K, V = (t.as_strided((n_pages, H, page, D), (step, page * D, D, 1)) for t in (big, big2))
    m = mirror([46], H, D, page, cap=48)
    m.table = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    Kh, Vh = rand((3, H, page, D), BF, 1), rand((3, H, page, D), BF, 2)
    K.copy_(Kh)
    V.copy_(Vh)
    m.K, m.V = Kh, Vh
    m.weight = torch.rand(3, H, page).double()
    m.pos = torch.zeros(3, H, page, dtype=torch.int32)
    m.dev = dict(K=K, V=V, weight=m.weight.float().cuda(), pos=m.pos.cuda(), table=m.table.cuda(), lens=m.lens.cuda(), seen=m.seen.cuda())
    check(m, [30], 4)


def test_binding_refuses_wrong_tensors():
    m = mirror([100], 2, 64, 16)
    cache = m.cache(ec)
    ws = scratch(ec.ec_paged_chunk_workspace(cache, 4))
    q, s = torch.zeros(30, 4, 64, dtype=BF, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros(30, 4, device="cuda")
    bad = [(q.half(), s, s, q, lse), (q, s.long(), s, q, lse), (q, s, s[:0], q, lse), (q, s, s, q[:29], lse), (q, s, s, q, lse[:, :3]),
           (q.cpu(), s, s, q, lse), (q, s, s, q, lse.double()), (q[:, :, ::2], s, s, q, lse), (q, s.cpu(), s, q, lse)]
    for a, st, c, o, z in bad:
        with pytest.raises((ValueError, ec.EcError)):
            ec.ec_paged_chunk_attention(a, st, c, cache, 0.125, o, z, ws)
    for kw in (dict(scale=0.0), dict(scale=float("nan")), dict(ws=ws[:256])):
        with pytest.raises(ec.EcError):
            ec.ec_paged_chunk_attention(q, s, s, cache, kw.get("scale", 0.125), torch.empty_like(q), lse, kw.get("ws", ws))
    with pytest.raises(ec.EcError):
        ec.ec_paged_chunk_weights(q, lse, s, s, cache, 0.125, 1.5, ws)
    with pytest.raises(ec.EcError):                            # not a multiple of the cache's heads
        ec.ec_paged_chunk_attention(q[:, :3], s, s, cache, 0.125, torch.empty_like(q[:, :3]), None, ws)
