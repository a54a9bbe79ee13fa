"""Pages handed out and taken back on the GPU, rotary positions, rows into the pages, and whole runs of a chunk."""
import math

import pytest
import torch

from chunk_reference import ChunkExact, PoolModel, rotary
from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200.session import PagedPoolSession
from test_paged_gpu import BF, HF, rand, scratch, state_of

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ pages

class Pool:
    """Random problems on a pool, on the device and as a model."""

    def __init__(self, N, page, spare, seed, most=60, gone=0.2, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        lens = torch.randint(0, most, (N,), generator=g).tolist()
        held = [-(-x // page) for x in lens]
        self.max_pages = max_pages or -(-2 * most // page) + 1
        n_pages = sum(held) + spare
        order = torch.randperm(n_pages, generator=g).tolist()
        table, at = [], 0
        for h in held:
            table.append(order[at:at + h] + [-1] * (self.max_pages - h))
            at += h
        for n in torch.nonzero(torch.rand(N, generator=g) < gone).flatten().tolist():
            lens[n] = -1 if n % 2 else lens[n] // 2              # over, or shrunk
        seen = [abs(x) + 7 * n for n, x in enumerate(lens)]
        self.model = PoolModel(lens, seen, held, table, order[at:], page)
        shape = (n_pages, 1, page, 64)
        K, V = (torch.zeros(shape, dtype=BF, device="cuda") for _ in range(2))
        self.lens, self.seen, self.held, self.table = i32(lens), i32(seen), i32(held), i32(table)
        self.free, self.n_free = i32(order[at:] + [-9] * at), i32([n_pages - at])
        self.state = scratch(ec.ec_paged_state_bytes(N))
        self.cache = ec.ec_paged_init(K, V, torch.zeros(shape[:3], device="cuda"), torch.zeros(shape[:3], dtype=torch.int32, device="cuda"),
                                      self.table, self.lens, self.seen, self.state)
        self.pages = ec.ec_pages(self.free, self.n_free, self.held)
        self.N = N

    def release(self):
        ec.ec_paged_release(self.cache, self.pages)
        self.model.release()
        self.compare()

    def reserve(self, counts, tokens, advance=True, limit=0):
        starts, granted = i32([-7] * (self.N + 1)), i32([-7] * self.N)
        slots, pos = (torch.full((tokens,), -7, dtype=torch.int32, device="cuda") for _ in range(2)) if advance else (None, None)
        ec.ec_paged_reserve(self.cache, self.pages, i32(counts), starts, granted, slots, pos, advance, limit)
        want = self.model.reserve(counts, tokens, advance, limit)
        assert granted.tolist() == want[1]
        if advance:
            assert starts.tolist() == want[0] and slots.tolist() == want[2] and pos.tolist() == want[3]
        self.compare()
        return want[1]

    def compare(self):
        m = self.model
        assert self.lens.tolist() == m.lens and self.seen.tolist() == m.seen and self.held.tolist() == m.held
        assert int(self.n_free) == len(m.free) and self.free[:len(m.free)].tolist() == m.free
        got = self.table.tolist()
        assert all(got[n][:h] == m.table[n][:h] for n, h in enumerate(m.held))
        assert ec.ec_device_status(self.state) == ec.EC_OK


@pytest.mark.parametrize("N,page,spare", [(1, 16, 5), (2, 1, 100), (33, 16, 200), (300, 4, 3000), (1024, 8, 4000), (1025, 16, 6000), (3000, 64, 5000)])
def test_pages_come_and_go(N, page, spare):
    p = Pool(N, page, spare, seed=N)
    g = torch.Generator().manual_seed(1)
    for step in range(3):
        p.release()
        counts = torch.randint(-1, 12, (N,), generator=g).tolist()
        p.reserve(counts, sum(max(c, 0) for c in counts) + (5 if step == 1 else 0))
    p.release()


@pytest.mark.parametrize("spare", [0, 1, 3, 7, 20])
def test_a_pool_that_runs_out_refuses_in_order(spare):
    p = Pool(50, 4, spare, seed=spare, gone=0.0)
    counts = [(3 * n) % 9 for n in range(50)]
    granted = p.reserve(counts, sum(counts))
    assert any(c and not g for c, g in zip(counts, granted)) and (spare == 0 or any(granted))


def test_refused_for_the_table_or_the_packed_rows():
    p = Pool(4, 4, 100, seed=2, most=20, gone=0.0, max_pages=6)
    p.reserve([25, 1, 100, 2], 200)                        # the table of problems 0 and 2 is too short
    p.reserve([2, 2, 3, 4], 6)                             # tokens of problems 2 and 3 lie behind the packed rows
    p.reserve([0, 0, 0, 0], 0)


def test_pages_alone_up_to_a_limit():
    p = Pool(40, 4, 400, seed=3, gone=0.1)
    before = p.lens.clone()
    p.reserve([1] * 40, 0, advance=False, limit=30)
    p.reserve([9] * 40, 0, advance=False)
    assert torch.equal(before, p.lens)
    p.release()


def test_pool_counts_out_of_range_are_reported():
    for spoil in (lambda p: p.n_free.fill_(-3), lambda p: p.n_free.fill_(1 << 20), lambda p: p.held.fill_(-1), lambda p: p.held.fill_(1000),
                  lambda p: p.free.fill_(1 << 20), lambda p: p.table.fill_(-5)):
        p = Pool(6, 4, 50, seed=4, gone=0.0)
        spoil(p)
        granted, slots = i32([0] * 6), i32([0] * 60)
        ec.ec_paged_reserve(p.cache, p.pages, i32([10] * 6), i32([0] * 7), granted, slots, i32([0] * 60))
        assert ec.ec_device_status(p.state) == ec.EC_ERR_PAGE or not granted.any()
        n_rows = p.cache.n_pages * 4
        assert ((slots >= -1) & (slots < n_rows)).all()
        p = Pool(6, 4, 50, seed=4, gone=0.5)
        spoil(p)
        ec.ec_paged_release(p.cache, p.pages)
        torch.cuda.synchronize()
        assert 0 <= int(p.n_free) <= p.cache.n_pages or int(p.n_free) in (-3, 1 << 20)


def test_rows_that_join_need_slots():
    p = Pool(6, 4, 50, seed=4)
    with pytest.raises(ValueError):
        ec.ec_paged_reserve(p.cache, p.pages, i32([1] * 6), None, i32([0] * 6))
    with pytest.raises(ValueError):
        ec.ec_paged_reserve(p.cache, p.pages, i32([1] * 6), None, i32([0] * 6), i32([0] * 6), i32([0] * 5))


def test_a_captured_reserve_replayed():
    p = Pool(20, 8, 600, seed=5)
    counts, tokens = [n % 5 for n in range(20)], 40
    c, starts, granted, slots, pos = i32(counts), i32([0] * 21), i32([0] * 20), i32([0] * tokens), i32([0] * tokens)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        ec.ec_paged_release(p.cache, p.pages)
        ec.ec_paged_reserve(p.cache, p.pages, c, starts, granted, slots, pos)
    for _ in range(4):
        g.replay()
        p.model.release()
        want = p.model.reserve(counts, tokens)
        torch.cuda.synchronize()
        assert granted.tolist() == want[1] and slots.tolist() == want[2] and pos.tolist() == want[3]
        p.compare()


# ------------------------------------------------------------------ rotary

def turn_tolerance(x, want, factor):
    """An angle is off by 2^-24 of a half turn and the sine by two steps of fp32, products and sum by three roundings; the result once.
    |a| + |b| <= 2 max|x| of the head."""
    half = torch.finfo(x.dtype).eps / 2
    top = x.double().abs().amax(-1, keepdim=True)
    return half * want.abs() + 2 * top * abs(factor) * (math.pi * 2.0 ** -24 + 6 * 2.0 ** -24) * (1 + half) + torch.finfo(x.dtype).tiny * half


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (64, 48, False), (64, 8, True), (128, 128, False), (128, 128, True),
                                               (128, 64, False), (128, 16, False), (128, 24, True), (128, 0, False)])
def test_rotary_both_ways(D, rot, interleaved, dt):
    freqs, factor = ec.ec_rotary_frequencies(max(rot, 2), scaling=ec.EC_ROTARY_BY_PARTS, stretch=4.0, trained=4096.0)
    freqs = freqs[:rot // 2] if rot else None
    for N, T, heads in ((1, 1, 1), (3, 70, 5), (2, 1100, 3)):
        x = rand((N, T, heads, D), dt, T)
        pos = torch.randint(0, 100000, (N, T), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
        for inverse in (False, True):
            out = torch.empty_like(x, device="cuda")
            ec.ec_rotary(x.cuda(), out, pos.cuda(), None if freqs is None else freqs.cuda(), rot, interleaved, factor, inverse)
            want = rotary(x, pos, freqs, factor, rot, interleaved, inverse) if rot else x.double()
            assert ((out.cpu().double() - want).abs() <= turn_tolerance(x, want, factor)).all()
            assert torch.equal(out.cpu()[..., rot:].view(torch.int16), x[..., rot:].view(torch.int16))     # the rest as it was, bit for bit


@pytest.mark.parametrize("N,T,heads,D,rot,interleaved", [(4300, 7, 1, 64, 64, False), (30011, 1, 1, 64, 48, False), (2, 14000, 3, 128, 24, True),
                                                         (1, 100, 300, 64, 32, True), (3, 11, 97, 128, 128, False), (1, 1, 2049, 64, 16, False)])
def test_rotary_many_tokens_of_few_heads_and_the_other_way_round(N, T, heads, D, rot, interleaved):
    """Tokens that share a CTA across problems, and heads of a token that several CTAs share."""
    freqs, factor = ec.ec_rotary_frequencies(rot)
    x = rand((N, T, heads, D), BF, 3)
    pos = torch.randint(0, 5000, (N, T), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    out = torch.full_like(x, 7.0, device="cuda")
    ec.ec_rotary(x.cuda(), out, pos.cuda(), freqs.cuda(), rot, interleaved, 1.25)
    want = rotary(x, pos, freqs, 1.25, rot, interleaved)
    assert ((out.cpu().double() - want).abs() <= turn_tolerance(x, want, 1.25)).all()
    assert torch.equal(out.cpu()[..., rot:].view(torch.int16), x[..., rot:].view(torch.int16))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_far_and_negative_positions(interleaved):
    freqs, _ = ec.ec_rotary_frequencies(64)
    pos = torch.tensor([0, 1, -1, 1 << 20, (1 << 24) + 1, 1 << 30, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32)
    x = rand((1, 8, 2, 64), HF, 1)
    out = torch.empty_like(x, device="cuda")
    ec.ec_rotary(x.cuda(), out, pos.cuda(), freqs.cuda(), 64, interleaved)
    # the oracle's own angles: 2^31 times the rounding of a frequency and of the product
    want = rotary(x, pos[None], freqs, 1.0, 64, interleaved)
    extra = 2 * x.double().abs().amax(-1, keepdim=True) * pos.double().abs()[None, :, None, None] * 2.0 ** -51
    assert ((out.cpu().double() - want).abs() <= turn_tolerance(x, want, 1.0) + extra).all()


def test_the_inverse_is_the_gradient():
    """<R x, y> = <x, R^T y>, and differences of a linear map are the map."""
    freqs, _ = ec.ec_rotary_frequencies(128)
    pos = torch.arange(50, dtype=torch.int32) * 1000
    x, y, d = (rand((1, 50, 4, 128), HF, s) for s in (1, 2, 3))

    def f(t, inverse=False):
        out = torch.empty_like(t, device="cuda")
        ec.ec_rotary(t.cuda(), out, pos.cuda(), freqs.cuda(), 128, False, 1.5, inverse)
        return out.cpu().double()
    n = x.numel()
    lhs, rhs = (f(x) * y.double()).sum(), (x.double() * f(y, True)).sum()
    assert abs(lhs - rhs) <= 2 * n * 2.0 ** -11 * 8
    step = (x.double() + d.double()).to(HF)
    diff = ((f(step) - f(x)) * y.double()).sum()
    lin = ((step.double() - x.double()) * f(y, True)).sum()
    assert abs(diff - lin) <= 3 * n * 2.0 ** -11 * 8


def test_rotary_strides_and_in_place():
    freqs, _ = ec.ec_rotary_frequencies(64)
    wide = torch.randn(3, 90, 10, 64, device="cuda").to(BF)
    x = wide[:, :, 2:6]
    before = wide.clone()
    pos = torch.arange(90, dtype=torch.int32, device="cuda") + 5
    dense = torch.empty(3, 4, 90, 64, dtype=BF, device="cuda")
    ec.ec_rotary(x, dense.transpose(1, 2), pos, freqs.cuda(), 64, False)                 # heads in front of tokens, positions for all
    ec.ec_rotary(x, x, pos, freqs.cuda(), 64, False)
    assert torch.equal(dense.transpose(1, 2), x)
    assert torch.equal(wide[:, :, :2], before[:, :, :2]) and torch.equal(wide[:, :, 6:], before[:, :, 6:])
    want = rotary(before[:, :, 2:6].cpu(), pos.cpu()[None].expand(3, 90), freqs, 1.0, 64, False)
    assert ((x.cpu().double() - want).abs() <= turn_tolerance(before[:, :, 2:6].cpu(), want, 1.0)).all()


def test_rotary_binding_refuses():
    x = torch.zeros(2, 3, 4, 64, dtype=BF, device="cuda")
    pos, f = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    for args in ((x.float(), x, pos, f, 64), (x, x[:1], pos, f, 64), (x, x.half(), pos, f, 64), (x, x, pos.long(), f, 64), (x, x, pos[:1], f, 64),
                 (x, x, pos, f[:31], 64), (x, x, pos, f.float(), 64), (x.cpu(), x, pos, f, 64), (x[..., ::2], x, pos, f, 64), (x[0], x, pos, f, 64)):
        with pytest.raises((ValueError, ec.EcError)):
            ec.ec_rotary(*args, False)


# ------------------------------------------------------------------ rows into the pages

@pytest.mark.parametrize("rows", ["heads", "tokens"])
@pytest.mark.parametrize("dt,D,rot,page,tokens", [(BF, 128, 128, 16, 40), (HF, 64, 32, 24, 7), (BF, 64, 0, 1, 3), (HF, 128, 64, 100, 2500)])
def test_join(dt, D, rot, page, tokens, rows):
    H, Hq = 3, 6
    m = PagedMirror([tokens + 3], H, D, page, tokens + 3, dt, rows)
    cache = m.cache(ec)
    freqs, factor = ec.ec_rotary_frequencies(max(rot, 2), scaling=ec.EC_ROTARY_LINEAR, stretch=2.0)
    freqs = freqs[:rot // 2].cuda() if rot else None
    both = rand((tokens, Hq + 2 * H, D), dt, 1)
    g = torch.Generator().manual_seed(2)
    row = torch.randperm(tokens + 3, generator=g)[:tokens]
    slots = (m.table[0].long()[row // page] * page + row % page).to(torch.int32)
    left_out = torch.rand(tokens, generator=g) < 0.2
    slots[left_out] = -1
    pos = torch.randint(0, 5000, (tokens,), generator=g, dtype=torch.int32)
    w = torch.rand(tokens, H, generator=g)
    dev = both.cuda()
    q_out = torch.full((tokens, Hq, D), 7.0, dtype=dt, device="cuda")
    ec.ec_paged_join(dev[:, :Hq], q_out, dev[:, Hq:Hq + H], dev[:, Hq + H:], w.cuda(), slots.cuda(), pos.cuda(), cache, freqs, rot, False, factor)
    turn = (lambda x: rotary(x, pos, freqs.cpu(), factor, rot, False)) if rot else (lambda x: x.double())
    want = turn(both[:, :Hq])
    near = (q_out.cpu().double() - want).abs() <= turn_tolerance(both[:, :Hq], want, factor)
    assert near[~left_out].all() and (q_out.cpu()[left_out] == 7.0).all()
    into = ~left_out
    p, s = slots.long()[into] // page, slots.long()[into] % page
    K, want_k = m.dev["K"].cpu(), turn(both[:, Hq:Hq + H])
    assert ((K[p, :, s].double() - want_k[into]).abs() <= turn_tolerance(both[:, Hq:Hq + H], want_k, factor)[into]).all()
    m.K[p, :, s] = K[p, :, s]                          # the rest of the pool has to be as it was, bit for bit
    m.V[p, :, s] = both[into][:, Hq + H:]
    m.weight[p, :, s] = w[into].double()
    m.pos[p, :, s] = pos[into][:, None].expand(-1, H)
    m.assert_same_rows(0.0, "join")


@pytest.mark.parametrize("H,Hq,tokens", [(1, 0, 30000), (1, 2, 20000), (5, 200, 37), (3, 150, 300), (40, 7, 2)])
def test_join_many_tokens_of_few_heads_and_the_other_way_round(H, Hq, tokens):
    """Tokens that share a CTA, and heads of a token that several CTAs share: every row, weight and position is written once."""
    D, page = 64, 16
    m = PagedMirror([tokens + 3], H, D, page, tokens + 3, BF, "heads")
    cache = m.cache(ec)
    freqs, _ = ec.ec_rotary_frequencies(64)
    both = rand((tokens, Hq + 2 * H, D), BF, 1)
    g = torch.Generator().manual_seed(2)
    row = torch.randperm(tokens + 3, generator=g)[:tokens]
    slots = (m.table[0].long()[row // page] * page + row % page).to(torch.int32)
    slots[::5] = -1
    pos = torch.randint(0, 5000, (tokens,), generator=g, dtype=torch.int32)
    w = torch.rand(tokens, H, generator=g)
    dev, into = both.cuda(), slots >= 0
    q_out = torch.full((tokens, Hq, D), 7.0, dtype=BF, device="cuda") if Hq else None
    ec.ec_paged_join(dev[:, :Hq] if Hq else None, q_out, dev[:, Hq:Hq + H], dev[:, Hq + H:], w.cuda(), slots.cuda(), pos.cuda(), cache,
                     freqs.cuda(), 64, False)
    want = rotary(both[:, :Hq + H], pos, freqs, 1.0, 64, False)
    allowed = turn_tolerance(both[:, :Hq + H], want, 1.0)
    if Hq:
        assert ((q_out.cpu().double() - want[:, :Hq]).abs() <= allowed[:, :Hq])[into].all() and (q_out.cpu()[~into] == 7.0).all()
    p, s = slots.long()[into] // page, slots.long()[into] % page
    K = m.dev["K"].cpu()
    assert ((K[p, :, s].double() - want[into][:, Hq:]).abs() <= allowed[into][:, Hq:]).all()
    m.K[p, :, s] = K[p, :, s]
    m.V[p, :, s] = both[into][:, Hq + H:]
    m.weight[p, :, s] = w[into].double()
    m.pos[p, :, s] = pos[into][:, None].expand(-1, H)
    m.assert_same_rows(0.0, "join")


def test_join_keys_alone_and_slots_out_of_range():
    m = PagedMirror([20], 2, 64, 16, 32)
    cache = m.cache(ec)
    k, v = rand((4, 2, 64), BF, 1), rand((4, 2, 64), BF, 2)
    n = m.K.shape[0] * 16
    slots = torch.tensor([n, 3, -5, (1 << 31) - 1], dtype=torch.int32)
    ec.ec_paged_join(None, None, k.cuda(), v.cuda(), None, slots.cuda(), i32([9, 8, 7, 6]), cache, None, 0, False)
    assert ec.ec_device_status(state_of(cache)) == ec.EC_ERR_PAGE
    m.K[0, :, 3], m.V[0, :, 3], m.weight[0, :, 3], m.pos[0, :, 3] = k[1], v[1], 0.0, 8
    m.assert_same_rows(0.0, "join")


# ------------------------------------------------------------------ whole runs

def mirror_of(s):
    """A host copy of a session's cache, as the reference takes it."""
    m = PagedMirror.__new__(PagedMirror)
    m.N, m.H, m.D, m.dtype, m.page = s.N, s.H, s.D, s.Kp.dtype, s.Kp.shape[2]
    m.max_pages = s.table.shape[1]
    m.K, m.V, m.weight, m.pos = s.Kp.cpu(), s.Vp.cpu(), s.weight.cpu().double(), s.pos.cpu()
    m.table, m.lens, m.seen = s.table.cpu(), s.lens.cpu(), s.seen.cpu()
    m.dev = dict(K=s.Kp, V=s.Vp, weight=s.weight, pos=s.pos, table=s.table, lens=s.lens, seen=s.seen)
    return m


@pytest.mark.parametrize("dt,D,G,interleaved", [(BF, 128, 4, False), (HF, 64, 3, True)])
def test_a_prompt_in_pieces_is_the_prompt_at_once(dt, D, G, interleaved):
    """Without eviction, pieces of prompts with rotary positions give causal attention of the turned rows."""
    N, H, T = 3, 2, 150
    freqs, factor = ec.ec_rotary_frequencies(D)
    s = PagedPoolSession(N, H, D, budget=400, recent=4, sinks=1, scale=D ** -0.5, pool_rows=N * 500, chunk=100, Hq=H * G, page_size=16,
                         dtype=dt, rot=D, interleaved=interleaved, freqs=freqs)
    q, k, v = rand((N, T, H * G, D), dt, 1), rand((N, T, H, D), dt, 2), rand((N, T, H, D), dt, 3)
    done = [0] * N
    got = torch.zeros(N, T, H * G, D, dtype=torch.float64)
    for counts in ([40, 1, 100], [0, 33, 50], [100, 64, 0], [10, 52, 0]):
        sel = [(n, done[n], c) for n, c in enumerate(counts)]
        part = [torch.cat([t[n, a:a + c] for n, a, c in sel]).cuda() for t in (q, k, v)]
        out = torch.empty_like(part[0])
        s.chunk(*part, i32(counts), out)
        at = 0
        for n, a, c in sel:
            got[n, a:a + c] = out[at:at + c].cpu().double()
            at += c
            done[n] += c
    assert s.status() == ec.EC_OK and done == [T] * N and s.lens.tolist() == [T] * N and s.seen.tolist() == [T] * N
    pos = torch.arange(T)
    half = torch.finfo(dt).eps / 2
    for n in range(N):
        qt, kt = rotary(q[n], pos, freqs, factor, D, interleaved).to(dt).double(), rotary(k[n], pos, freqs, factor, D, interleaved).to(dt).double()
        for i in range(H * G):
            x = (qt[:, i] @ kt[:, i // G].T) * D ** -0.5
            x = x.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -math.inf)
            p = torch.softmax(x, -1)
            want = p @ v[n, :, i // G].double()
            # a turned row may round the other way: half a step of its type, two of them in a score
            rows = (qt[:, i].abs() @ kt[:, i // G].abs().T) * D ** -0.5
            tol = half * want.abs() + (half + 4 * half * rows.amax(-1, keepdim=True) + 2.0 ** -10) * (p @ v[n, :, i // G].double().abs())
            assert ((got[n, :, i] - want).abs() <= tol).all()
    # positions of the rows, and that every problem has pages of its own
    m = mirror_of(s)
    for n in range(N):
        page, slot = m.where(n, T)
        assert torch.equal(m.pos[page, 0, slot], torch.arange(T, dtype=torch.int32))
    held = [p for n in range(N) for p in s.table[n, :int(s.pages.held[n])].tolist()]
    assert len(set(held)) == len(held) and len(held) + int(s.pages.n_free) == s.Kp.shape[0]


def test_a_chunk_evicts_as_the_definition_does():
    """Call by call: the rows that stay are those that the gathered weights say."""
    N, H, D, G, budget = 3, 2, 64, 2, 64
    s = PagedPoolSession(N, H, D, budget=budget, recent=8, sinks=2, scale=0.125, pool_rows=N * 160, chunk=90, Hq=H * G, page_size=16, decay=0.97)
    ws, app = scratch(ec.ec_paged_chunk_workspace(s.cache, H * G)), scratch(ec.ec_paged_append_workspace(s.cache, 0, budget))
    for step, counts in enumerate(([90, 10, 30], [5, 60, 1], [1, 0, 80], [33, 33, 33])):
        tokens = sum(counts)
        q, k, v = rand((tokens, H * G, D), BF, 10 + step), rand((tokens, H, D), BF, 20 + step), rand((tokens, H, D), BF, 30 + step)
        slots, pos = torch.empty(tokens, dtype=torch.int32, device="cuda"), torch.empty(tokens, dtype=torch.int32, device="cuda")
        ec.ec_paged_release(s.cache, s.pages)
        ec.ec_paged_reserve(s.cache, s.pages, i32(counts), s.starts, s.granted, slots, pos)
        turned = torch.empty(tokens, H * G, D, dtype=BF, device="cuda")
        ec.ec_paged_join(q.cuda(), turned, k.cuda(), v.cuda(), None, slots, pos, s.cache, None, 0, False)
        m = mirror_of(s)
        out, lse = torch.empty_like(turned), torch.empty(tokens, H * G, device="cuda")
        ec.ec_paged_chunk_attention(turned, s.starts, s.granted, s.cache, s.scale, out, lse, ws)
        ec.ec_paged_chunk_weights(turned, lse, s.starts, s.granted, s.cache, s.scale, s.decay, ws)
        c = torch.tensor(counts)
        ChunkExact(m, q, s.starts.cpu(), c, s.scale).assert_out(out, lse, f"step {step}")
        ChunkExact(m, q, s.starts.cpu(), c, s.scale, s.decay, lse=lse.cpu()).assert_weights(s.weight, f"step {step}")
        m = mirror_of(s)                                   # eviction goes by the weights that are there
        ec.ec_paged_append(None, None, None, None, None, s.cache, False, budget, s.recent, s.sinks, app)
        none = torch.zeros(N, H, 0, D)
        m.append(none, none, None, None, None, 0, False, budget, s.recent, s.sinks)
        m.assert_same_rows(0.0, f"step {step}")
        assert s.status() == ec.EC_OK and max(s.lens.tolist()) <= budget


def test_steps_after_chunks_and_a_pool_that_runs_out():
    """Sequences come and go in a pool that cannot hold all of them at their budget."""
    N, H, D, budget, page = 6, 2, 64, 48, 16
    s = PagedPoolSession(N, H, D, budget=budget, recent=8, sinks=1, scale=0.125, pool_rows=12 * page, chunk=32, page_size=page)
    counts = [32, 16, 20, 1, 30, 31]
    q, k, v = rand((sum(counts), H, D), BF, 1).cuda(), rand((sum(counts), H, D), BF, 2).cuda(), rand((sum(counts), H, D), BF, 3).cuda()
    out = torch.full_like(q, 7.0)
    s.chunk(q, k, v, i32(counts), out)
    assert s.granted.tolist() == counts and int(s.pages.n_free) == 12 - (2 + 1 + 2 + 1 + 2 + 2)
    one = [rand((N, H, D), BF, 4 + i).cuda() for i in range(3)]
    res = torch.empty_like(one[0])
    for step in range(20):
        s.decode(*one, res)
        assert s.status() == ec.EC_OK
        held = [p for n in range(N) for p in s.table[n, :int(s.pages.held[n])].tolist()]
        assert len(set(held)) == len(held) and len(held) + int(s.pages.n_free) == 12
    lens, granted = s.lens.tolist(), s.granted.tolist()
    assert max(lens) <= budget and 0 in granted and 1 in granted
    for n in range(N):
        assert (res[n] == 0).all().item() == (granted[n] == 0)
    stuck = granted.index(0)
    s.end((stuck + 1) % N)                                 # its pages go to those who waited
    s.decode(*one, res)
    assert s.granted.tolist()[stuck] == 1 and s.lens.tolist()[stuck] == lens[stuck] + 1
    s.begin((stuck + 1) % N)
    s.end((stuck + 2) % N)
    c = [0] * N
    c[(stuck + 1) % N] = 20
    s.chunk(q[:20], k[:20], v[:20], i32(c), out[:20])
    assert s.lens.tolist()[(stuck + 1) % N] == 20 and s.seen.tolist()[(stuck + 1) % N] == 20 and s.status() == ec.EC_OK


def test_a_captured_chunk_and_step():
    """One graph of a chunk and a step, replayed: the same as calls made one by one."""
    def make():
        return PagedPoolSession(2, 2, 64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=400, chunk=40, Hq=4, page_size=16)
    a, b = make(), make()
    tokens = 50
    q, k, v = rand((tokens, 4, 64), BF, 1).cuda(), rand((tokens, 2, 64), BF, 2).cuda(), rand((tokens, 2, 64), BF, 3).cuda()
    one = rand((2, 4, 64), BF, 4).cuda(), rand((2, 2, 64), BF, 5).cuda(), rand((2, 2, 64), BF, 6).cuda()
    counts = i32([30, 20])
    outs = [(torch.zeros_like(q), torch.zeros_like(one[0])) for _ in range(2)]

    def step(s, out, res):
        s.chunk(q, k, v, counts, out)
        s.decode(*one, res)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(a, *outs[0])                                  # once outside of the capture
        step(b, *outs[1])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(a, *outs[0])
        for c in ([30, 20], [0, 40], [7, 1], [40, 10]):
            counts.copy_(i32(c))
            g.replay()
            step(b, *outs[1])
            torch.cuda.synchronize()
            assert torch.equal(a.lens, b.lens) and torch.equal(a.seen, b.seen) and torch.equal(a.pages.held, b.pages.held)
            assert torch.equal(outs[0][1], outs[1][1])
            for n, length in enumerate(a.lens.tolist()):       # what lies behind the rows was never written
                rows = torch.arange(length, device="cuda")
                at = [(x.table[n].long()[rows // 16], rows % 16) for x in (a, b)]
                assert torch.equal(*(t[0] for t in at))
                for x, y in ((a.Kp, b.Kp), (a.Vp, b.Vp), (a.weight, b.weight), (a.pos, b.pos)):
                    assert torch.equal(x[at[0][0], :, at[0][1]], y[at[1][0], :, at[1][1]])
            assert torch.equal(outs[0][0][:sum(c)], outs[1][0][:sum(c)])


def test_the_session_refuses():
    s = PagedPoolSession(2, 2, 64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=400, chunk=40)
    with pytest.raises(ValueError):
        s.prompt(None, None, None)
    with pytest.raises(ValueError):
        s.append(torch.zeros(2, 2, 3, 64, dtype=BF, device="cuda"), None, None, fresh=True)
    q = torch.zeros(5, 2, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        s.chunk(q, q[:4], q, i32([5, 0]), torch.empty_like(q))
    with pytest.raises(ValueError):
        s.chunk(q, q, q, i32([5]), torch.empty_like(q))


def test_a_refused_call_leaves_the_session_as_it_was():
    """Wrong tensors are found before any row joins, and places that wait for pages keep their rows."""
    s = PagedPoolSession(2, 2, 64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=32, chunk=40, page_size=16)
    q = rand((32, 2, 64), BF, 1).cuda()
    out = torch.empty_like(q)
    s.chunk(q, q, q, i32([16, 16]), out)                   # the pool is empty now
    wide = torch.zeros(32, 2, 68, dtype=BF, device="cuda")[:, :, :64]
    for bad in (dict(k=q[:4]), dict(v=q.half()), dict(out=out[:, :1]), dict(q=wide), dict(out=wide), dict(counts=i32([16])),
                dict(lse=torch.empty(32, 1, device="cuda")), dict(k=q.cpu())):
        a = dict(q=q, k=q, v=q, counts=i32([16, 16]), out=out, lse=None)
        a.update(bad)
        with pytest.raises(ValueError):
            s.chunk(**a)
        assert s.lens.tolist() == [16, 16] and s.seen.tolist() == [16, 16] and s.pages.held.tolist() == [1, 1]
    one = q[:2].clone()
    with pytest.raises(ValueError):
        s.decode(one, one, one[:1], torch.empty_like(one))
    assert s.lens.tolist() == [16, 16]
    with pytest.raises(ValueError):
        s.append(torch.zeros(2, 2, 3, 32, dtype=BF, device="cuda"), torch.zeros(2, 2, 3, 64, dtype=BF, device="cuda"), None)
    assert s.lens.tolist() == [16, 16] and s.status() == ec.EC_OK
    for kw in (dict(scale=0.0), dict(decay=1.5), dict(rot=24), dict(rot=32), dict(rot=128), dict(rot=32, freqs=torch.ones(8))):
        with pytest.raises(ValueError):
            PagedPoolSession(**{**dict(N=2, H=2, D=64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=400, chunk=40), **kw})


def test_a_chunk_of_no_tokens():
    s = PagedPoolSession(2, 2, 64, budget=64, recent=8, sinks=1, scale=0.125, pool_rows=400, chunk=40)
    q = rand((5, 2, 64), BF, 1).cuda()
    s.chunk(q, q, q, i32([2, 3]), torch.empty_like(q))
    weight = s.weight.clone()
    s.chunk(q[:0], q[:0], q[:0], i32([0, 0]), torch.empty_like(q[:0]))
    s.chunk(q[:0], q[:0], q[:0], i32([4, 0]), torch.empty_like(q[:0]))   # no packed rows for them: not granted
    assert s.lens.tolist() == [2, 3] and s.granted.tolist() == [0, 0] and torch.equal(s.weight, weight) and s.status() == ec.EC_OK
    x = torch.empty(2, 0, 4, 64, dtype=BF, device="cuda")
    ec.ec_rotary(x, x, torch.empty(2, 0, dtype=torch.int32, device="cuda"), ec.ec_rotary_frequencies(64)[0].cuda(), 64, False)
