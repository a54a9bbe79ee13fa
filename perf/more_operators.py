"""Operators of a chunk of new tokens on a paged cache, with their plain forms.

A serving step takes several new tokens of many sequences at once: a piece of a prompt, a whole prompt, a few drafted tokens to
be verified. The tokens of all problems lie one after the other ("packed"): problem n has counts[n] tokens from starts[n] on.

  reserve    pages of problems that ended or shrank come back to the pool's stack of free pages, then the chunk's rows get theirs:
             block table, and for every token the slot of its row (page * page_size + place, -1: none) and its position
  join       rotary positions on the chunk's queries and keys, keys and values into the slots
  rotary     rotary positions alone, forward or backward (the transposed rotation, which is its gradient)
  attention  token t of problem n sees the rows 0 .. lens[n] - counts[n] + t of its problem, its own the last of them:
                 out = softmax(scale * q K^T) V,   lse = log sum exp(scale * q K^T)
  weights    what every row received from the chunk's queries joins its gathered weight:
                 weight_j <- decay^count weight_j + sum_t decay^(count - 1 - t) sum_g p[t, g, j]

Rotary: pair i of a head turns by the angle position * freq_i, both of its elements times `factor`:
(a, b) -> (a cos - b sin, a sin + b cos). Pairs are the elements (2 i, 2 i + 1) or (i, i + rot / 2) of the first `rot`.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
DECAY = 0.998


def listed():
    return [
        # eight users in the middle of their prompts: nothing but latency
        dict(name="reserve few", op="reserve", N=8, T=48, L=700, page=16, ended=0.0),
        # a full server: 512 places, some of which have just ended, and a prompt piece for many
        dict(name="reserve many", op="reserve", N=512, T=96, L=4096, page=16, ended=0.1),
        # drafted tokens of six users, interleaved pairs, half of a head turns
        dict(name="join drafted", op="join", N=6, T=4, L=2000, H=8, G=4, D=128, rot=64, pairs="next", page=16, dtype="fp16", rows="heads", stretch=1.0),
        # prompts of four users, grouped heads, out of one projection's output, stretched context
        dict(name="join prompts", op="join", N=4, T=2048, L=0, H=8, G=4, D=128, rot=128, pairs="half", page=64, dtype="bf16", rows="tokens", stretch=8.0),
        # the gradient of a layer's queries
        dict(name="rotary back", op="rotary", N=2, T=4096, L=0, H=32, D=128, rot=128, pairs="half", dtype="bf16", stretch=1.0, back=True),
        # drafted tokens of 32 users looked over at once: bandwidth
        dict(name="attention drafted", op="attention", N=32, T=8, L=8192, H=8, G=4, D=128, page=64, dtype="bf16", rows="heads"),
        # a serving batch: pieces of prompts of all lengths on contexts of all lengths
        dict(name="attention mixed", op="attention", N=16, T=512, L=4096, H=8, G=4, D=128, page=16, dtype="bf16", rows="tokens"),
        # odd group, odd pages, smaller heads, half precision
        dict(name="attention odd", op="attention", N=7, T=203, L=3001, H=5, G=7, D=64, page=24, dtype="fp16", rows="heads"),
        # one long prompt at once: the tensor cores
        dict(name="attention prompt 8192", op="attention", N=1, T=8192, L=8192, H=8, G=4, D=128, page=64, dtype="bf16", rows="heads"),
        # the weights that go with the drafted tokens, the odd batch and the long prompt
        dict(name="weights drafted", op="weights", N=32, T=8, L=8192, H=8, G=4, D=128, page=64, dtype="bf16", rows="heads"),
        dict(name="weights odd", op="weights", N=7, T=203, L=3001, H=5, G=7, D=64, page=24, dtype="fp16", rows="heads"),
        dict(name="weights prompt 8192", op="weights", N=1, T=8192, L=8192, H=8, G=4, D=128, page=64, dtype="bf16", rows="heads"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["reserve", "join", "rotary", "attention", "attention", "attention", "weights", "weights"])
    if op == "reserve":
        N = _log(rng, 1, 512)
        return dict(op=op, N=N, T=_log(rng, 1, min(8192, 49152 // N)), L=_log(rng, 16, 4096), page=rng.choice([1, 8, 16, 24, 64, 100, 128]),
                    ended=rng.choice([0.0, 0.1, 0.3]))
    c = dict(op=op, H=rng.choice([1, 2, 4, 5, 8, 16, 32]), D=rng.choice([64, 128]), dtype=rng.choice(["bf16", "fp16"]))
    if op in ("join", "rotary"):
        c["N"] = _log(rng, 1, 32)
        c["rot"] = rng.choice([c["D"], c["D"], c["D"] // 2, 48])
        c.update(pairs=rng.choice(["next", "half"]), stretch=rng.choice([1.0, 4.0, 32.0]))
        if op == "rotary":
            c.update(T=_log(rng, 1, min(16384, (1 << 25) // (c["N"] * c["H"] * c["D"]))), L=_log(rng, 1, 1000000), back=rng.random() < 0.5)
            return c
        c.update(G=rng.choice([1, 2, 3, 4, 8]), page=rng.choice([8, 16, 24, 64, 100, 128]), rows=rng.choice(["heads", "tokens"]))
        c["T"] = _log(rng, 1, min(8192, (1 << 25) // (c["N"] * c["H"] * c["G"] * c["D"])))
        c["L"] = rng.choice([0, _log(rng, 1, 2000)])
        return c
    c.update(G=rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]), page=rng.choice([8, 16, 24, 64, 100, 128]), rows=rng.choice(["heads", "tokens"]))
    c["N"] = _log(rng, 1, 32)
    c["T"] = _log(rng, 1, 4096)
    heads = c["N"] * c["H"] * c["G"]
    c["T"] = max(1, min(c["T"], int(math.sqrt((1 << 30) // heads))))
    c["L"] = c["T"] + _log(rng, 1, max(1, min(32768, (1 << 30) // (heads * c["T"]) - c["T"])))
    c["L"] = max(c["T"], min(c["L"], (1 << 29) // (c["N"] * c["H"] * c["D"])))
    return c


# ------------------------------------------------------------------ shapes that a case fixes

def _counts(case):
    """New tokens of every problem; part of the case, not of its seed."""
    N, T = case["N"], case["T"]
    r = random.Random(13 * N + T)
    got = [T] + [_log(r, 1, T) for _ in range(N - 1)]
    if case["op"] == "join" and case["L"] == 0:
        got = [T] * N                                       # whole prompts side by side
    if N > 3:
        got[2] = 0                                          # nothing new for this one
    return got


def _lens(case):
    """Rows of every problem, the chunk's among them (reserve, join: before they join)."""
    N, L = case["N"], case["L"]
    r = random.Random(17 * N + L)
    more = [_log(r, 1, max(1, L)) if L else 0 for _ in range(N)]
    if case["op"] in ("attention", "weights"):
        cnt = _counts(case)
        got = [L] + [c + min(L - c, x) for c, x in zip(cnt[1:], more[1:])]
        if N > 4:
            got[3] = cnt[3]                                 # a prompt's first piece
    else:
        got = more
    return got


def work(case):
    N, op = case["N"], case["op"]
    cnt, lens = _counts(case), _lens(case)
    tokens = sum(cnt)
    if op == "reserve":
        pages = -(-tokens // case["page"])
        return {"bytes": 4 * (7 * N + 2 * tokens + 2 * pages), "flops": tokens}
    H, D = case["H"], case["D"]
    if op == "rotary":
        n = N * case["T"] * H * D
        return {"bytes": 4 * n + 4 * N * case["T"], "flops": 3 * n}
    G = case["G"]
    if op == "join":
        return {"bytes": tokens * (4 * D * (H * G + 2 * H) + 8 + 8 * H), "flops": 3 * tokens * D * H * (G + 1)}
    seen = sum(c * (n - c) + c * (c + 1) // 2 for c, n in zip(cnt, lens))     # (token, row) pairs
    rows = sum(n for c, n in zip(cnt, lens) if c > 0)
    if op == "attention":
        return {"bytes": 4 * rows * H * D + 4 * tokens * H * G * D + 4 * tokens * H * G, "flops": 4 * D * H * G * seen}
    return {"bytes": rows * H * (2 * D + 8) + tokens * H * G * (2 * D + 4), "flops": 2 * D * H * G * seen}


# ------------------------------------------------------------------ inputs

def _freqs(rot, stretch):
    """Frequencies of the pairs: base 10000, the slow ones of a stretched context slowed down, the fast ones left."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * i / rot)
    if stretch == 1.0:
        return f, 1.0

    def pair_of(turns):                                     # the pair that turns this often over 4096 positions
        return rot * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))
    lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rot - 1)
    ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
    return f / stretch * ramp + f * (1 - ramp), 0.1 * math.log(stretch) + 1.0


def _prepare_reserve(case, seed):
    N, T, ps = case["N"], case["T"], case["page"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    lens, cnt = _lens(case), _counts(case)
    max_pages = -(-(max(x + c for x, c in zip(lens, cnt))) // ps)
    held = [-(-x // ps) for x in lens]
    ended = [r.random() < case["ended"] for _ in range(N)]
    grown = sum(-(-(x + c) // ps) for x, c in zip(lens, cnt))
    n_pages = grown + 5
    s = {"case": case, "tokens": sum(cnt)}
    # one buffer: lens, seen, held, the stack's height, the stack, the table
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    h = torch.tensor(held, device="cuda")
    at = torch.arange(max_pages, device="cuda")
    first = h.cumsum(0) - h
    table = torch.where(at[None] < h[:, None], perm[(first[:, None] + at).clamp(max=n_pages - 1)], -1)
    used = int(sum(held))
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_pages - used] = perm[used:]
    now = torch.tensor([-1 if e else x for e, x in zip(ended, lens)], dtype=torch.int32, device="cuda")
    seen = torch.tensor(lens, dtype=torch.int32, device="cuda") + torch.randint(0, 1000, (N,), generator=g, device="cuda", dtype=torch.int32)
    s["before"] = torch.cat([now, seen, h.to(torch.int32), torch.tensor([n_pages - used], dtype=torch.int32, device="cuda"), free,
                             table.to(torch.int32).flatten()])
    s["buffer"] = s["before"].clone()
    cut = [N, N, N, 1, n_pages, N * max_pages]
    s["lens"], s["seen"], s["held"], s["n_free"], s["free"], flat = s["buffer"].split(cut)
    s["table"] = flat.view(N, max_pages)
    s["counts"] = torch.tensor([0 if e else c for e, c in zip(ended, cnt)], dtype=torch.int32, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    s["starts"], s["granted"] = torch.empty(N + 1, **i32), torch.empty(N, **i32)
    s["slots"], s["positions"] = torch.empty(s["tokens"], **i32), torch.empty(s["tokens"], **i32)
    s["shape"] = (n_pages, 1, ps, 64)
    s["K"], s["V"] = (torch.zeros(s["shape"], dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s["weight"], s["pos"] = torch.zeros(s["shape"][:3], device="cuda"), torch.zeros(s["shape"][:3], **i32)
    return s


def prepare(case, seed):
    op, N = case["op"], case["N"]
    if op == "reserve":
        s = _prepare_reserve(case, seed)
    else:
        H, D, dt = case["H"], case["D"], DTYPES[case["dtype"]]
        g = torch.Generator(device="cuda").manual_seed(seed)
        s = {"case": case}

        def normal(*shape):
            return torch.randn(shape, generator=g, device="cuda", dtype=dt)
        if op in ("join", "rotary"):
            freqs, s["factor"] = _freqs(case["rot"], case["stretch"])
            s["freqs"] = freqs.cuda()
        if op == "rotary":
            s["x"] = normal(N, case["T"], H, D)
            s["out"] = torch.empty_like(s["x"])
            s["positions"] = (case["L"] + torch.arange(case["T"], device="cuda", dtype=torch.int32))[None] + torch.randint(
                0, 50, (N, 1), generator=g, device="cuda", dtype=torch.int32)
            return s
        ps, G = case["page"], case["G"]
        lens, cnt = _lens(case), _counts(case)
        full = [x + (c if op == "join" else 0) for x, c in zip(lens, cnt)]
        max_pages = max(1, -(-max(full) // ps))
        n_pages = N * max_pages + 3
        tokens = sum(cnt)
        shape = (n_pages, H, ps, D)

        def pool():
            return normal(*shape) if case["rows"] == "heads" else normal(n_pages, ps, H, D).permute(0, 2, 1, 3)
        s["K"], s["V"] = pool(), pool()
        s["table"] = torch.randperm(n_pages, generator=g, device="cuda")[:N * max_pages].view(N, max_pages).to(torch.int32)
        s["lens"] = torch.tensor(full, dtype=torch.int32, device="cuda")
        s["counts"] = torch.tensor(cnt, dtype=torch.int32, device="cuda")
        s["starts"] = (s["counts"].cumsum(0) - s["counts"]).to(torch.int32)
        s["seen"] = s["lens"] + 100
        s["pos"] = torch.full(shape[:3], -1, dtype=torch.int32, device="cuda")
        s["weight"] = torch.rand(shape[:3], generator=g, device="cuda")
        # every token's problem and its place in the chunk
        owner = torch.repeat_interleave(torch.arange(N, device="cuda"), s["counts"].long())
        t = torch.arange(tokens, device="cuda") - s["starts"].long()[owner]
        if op == "join":
            # out of one projection: queries, keys and values of a token side by side
            both = normal(tokens, H * (G + 2), D)
            s["q"], s["k"], s["v"] = both[:, :H * G], both[:, H * G:H * (G + 1)], both[:, H * (G + 1):]
            s["q_out"] = torch.empty(tokens, H * G, D, dtype=dt, device="cuda")
            row = s["lens"].long()[owner] - s["counts"].long()[owner] + t
            s["slots"] = (s["table"].long()[owner, row // ps] * ps + row % ps).to(torch.int32)
            s["positions"] = (row + 100).to(torch.int32)
        else:
            # heavy hitters: every key has a share of one direction that all queries of its head look along
            u = torch.randn(H, D, generator=g, device="cuda")
            u = (u / u.norm(dim=-1, keepdim=True)).to(dt)
            s["K"].add_((1.5 * torch.randn(n_pages, H, ps, 1, generator=g, device="cuda").abs()).to(dt) * u[None, :, None, :])
            s["q"] = normal(tokens, H * G, D).add_((math.sqrt(D) * u).to(dt).repeat_interleave(G, 0))
            s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(tokens, H * G, device="cuda")
            if op == "weights":
                s["before"] = s["weight"].clone()
                s["padded"] = _padded(s)
                x = _scores(s, s["padded"])
                s["lse"].copy_(_pack(s, torch.logsumexp(x, -1)))
                del x
    if own:
        from paper_2407_18121_b200 import binding as ec
        state = torch.empty(ec.ec_paged_state_bytes(N), dtype=torch.uint8, device="cuda")
        s["cache"] = ec.ec_paged_init(s["K"], s["V"], s["weight"], s["pos"], s["table"], s["lens"], s["seen"], state)
        if op == "reserve":
            s["pages"] = ec.ec_pages(s["free"], s["n_free"], s["held"])
        elif op in ("attention", "weights"):
            s["ws"] = torch.empty(ec.ec_paged_chunk_workspace(s["cache"], H * G), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms

def _release_and_reserve(s):
    c = s["case"]
    N, ps, max_pages, T = c["N"], c["page"], s["table"].shape[1], s["tokens"]
    at = torch.arange(max_pages, device="cuda")
    stack = torch.arange(s["free"].shape[0], device="cuda")
    # pages behind the last row of a problem come back, problem by problem
    held = s["held"].long()
    keep = torch.minimum(held, (s["lens"].long().clamp(min=0) + ps - 1) // ps)
    back = held - keep
    before = back.cumsum(0) - back
    gone = (at[None] >= keep[:, None]) & (at[None] < held[:, None])
    height = s["n_free"].long()
    place = height + before[:, None] + at[None] - keep[:, None]
    free = torch.cat([s["free"], s["free"][:1]])
    free.scatter_(0, torch.where(gone, place, stack.shape[0]).flatten(), s["table"].flatten())
    height = height + back.sum()
    held = keep
    # the chunk's pages come off the top
    lens, cnt = s["lens"].long(), s["counts"].long().clamp(min=0)
    ends = cnt.cumsum(0)
    fits = (lens >= 0) & (lens + cnt <= max_pages * ps) & (ends <= T)
    need = torch.where(fits & (cnt > 0), ((lens + cnt + ps - 1) // ps - held).clamp(min=0), 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= height))
    need_ok = torch.where(ok, need, 0)
    i = at[None] - held[:, None]
    new = (i >= 0) & (i < need_ok[:, None])
    source = (height - 1 - (upto - need)[:, None] - i).clamp(0, stack.shape[0] - 1)
    table = torch.where(new, free[source], s["table"])
    t = torch.arange(T, device="cuda")
    owner = torch.searchsorted(ends, t, right=True).clamp(max=N - 1)
    t_in = t - (ends - cnt)[owner]
    row = lens[owner] + t_in
    there = ok[owner] & (t_in < cnt[owner])
    page = table[owner, (row // ps).clamp(0, max_pages - 1)].long()
    s["slots"].copy_(torch.where(there, page * ps + row % ps, -1))
    s["positions"].copy_(torch.where(there, s["seen"].long()[owner] + t_in, -1))
    granted = torch.where(ok, cnt, 0)
    s["starts"][1:].copy_(ends)
    s["starts"][:1].zero_()
    s["granted"].copy_(granted)
    s["table"].copy_(table)
    s["free"].copy_(free[:-1])
    s["n_free"].copy_(height - need_ok.sum())
    s["held"].copy_(held + need_ok)
    s["lens"].copy_(lens + granted)
    s["seen"].add_(granted.to(torch.int32))


def _turn(x, positions, freqs, factor, rot, pairs, back):
    """x [..., heads, D], positions [...]: in 32 bits, the angles in 64."""
    angle = positions.double()[..., None, None] * freqs
    cos, sin = (torch.cos(angle) * factor).float(), (torch.sin(angle) * factor).float()
    if back:
        sin = -sin
    x = x.float()
    head, rest = x[..., :rot], x[..., rot:]
    if pairs == "next":
        a, b = head[..., 0::2], head[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)
    a, b = head[..., :rot // 2], head[..., rot // 2:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)


def _join(s):
    c = s["case"]
    how = (s["positions"], s["freqs"], s["factor"], c["rot"], c["pairs"], False)
    s["q_out"].copy_(_turn(s["q"], *how))
    page, place = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
    s["K"][page, :, place] = _turn(s["k"], *how).to(s["K"].dtype)
    s["V"][page, :, place] = s["v"]
    s["weight"][page, :, place] = 0.0
    s["pos"][page, :, place] = s["positions"][:, None].expand(-1, c["H"])


def _padded(s):
    """Rows and tokens of every problem side by side: (page, slot) of the rows, places of the tokens, what sees what."""
    c = s["case"]
    r = torch.arange(c["L"], device="cuda")
    t = torch.arange(c["T"], device="cuda")
    page, slot = s["table"].long()[:, (r // c["page"]).clamp(max=s["table"].shape[1] - 1)], (r % c["page"])[None].expand(c["N"], -1)
    token = (s["starts"].long()[:, None] + t).clamp(max=s["q"].shape[0] - 1)
    here = t[None] < s["counts"][:, None]
    limit = (s["lens"] - s["counts"])[:, None] + t                                              # [N, T]
    sees = (r[None, None] <= limit[..., None]) & here[..., None]                                # [N, T, L]
    return page, slot, token, here, sees


def _scores(s, padded):
    c = s["case"]
    N, H, G, D, T, L = (c[k] for k in ("N", "H", "G", "D", "T", "L"))
    page, slot, token, here, sees = padded
    K = s["K"][page, :, slot].float().transpose(1, 2)                                           # [N, H, L, D]
    q = s["q"][token].float().view(N, T, H, G, D).permute(0, 2, 3, 1, 4).reshape(N, H, G * T, D)
    x = (q @ K.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(N, H, G, T, L)
    return x.masked_fill_(~sees[:, None, None], -math.inf)


def _pack(s, y):
    """[N, H, G, T, ...] -> [tokens, H * G, ...]"""
    c = s["case"]
    t = torch.arange(c["T"], device="cuda")
    here = t[None] < s["counts"][:, None]
    y = y.movedim(3, 1)                                                                         # [N, T, H, G, ...]
    return y[here].flatten(1, 2)


def _attention(s):
    c = s["case"]
    N, H, G, D, T, L = (c[k] for k in ("N", "H", "G", "D", "T", "L"))
    padded = _padded(s)
    page, slot, token, here, sees = padded
    x = _scores(s, padded)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = x.sub_(m).exp_()
    z = e.sum(-1, keepdim=True)
    V = s["V"][page, :, slot].float().transpose(1, 2)                                           # [N, H, L, D]
    o = (e.view(N, H, G * T, L) @ V).view(N, H, G, T, D) / torch.where(z == 0, torch.ones_like(z), z)
    s["out"].copy_(_pack(s, o))
    s["lse"].copy_(_pack(s, (torch.log(z) + m)[..., 0]))


def _weights(s):
    c = s["case"]
    N, H, G, D, T, L = (c[k] for k in ("N", "H", "G", "D", "T", "L"))
    padded = _padded(s)
    page, slot, token, here, sees = padded
    x = _scores(s, padded)
    lse = s["lse"][token].view(N, T, H, G).permute(0, 2, 3, 1)[..., None]
    p = x.sub_(lse).exp_()
    t = torch.arange(T, device="cuda")
    left = (s["counts"][:, None] - 1 - t).clamp(min=0).double()                                 # [N, T]
    share = torch.where(here, torch.pow(torch.tensor(DECAY, dtype=torch.float64, device="cuda"), left), 0.0).float()
    gain = (share[:, None, None, None, :] @ p.nan_to_num_(0.0, 0.0, 0.0))[..., 0, :].sum(2)     # [N, H, L]
    held = torch.arange(L, device="cuda")[None] < torch.where(s["counts"] > 0, s["lens"], 0)[:, None]
    old = s["weight"][page, :, slot]                                                            # [N, L, H]
    kept = torch.pow(torch.tensor(DECAY, dtype=torch.float64, device="cuda"), s["counts"].double()).float()[:, None, None]
    fresh = torch.where(held[..., None], kept * old + gain.transpose(1, 2), old)
    # rows that no problem holds write nothing: their page is not theirs
    s["weight"].view(-1).scatter_(0, ((page[..., None] * H + torch.arange(H, device="cuda")) * c["page"] + slot[..., None])[held].flatten(),
                                  fresh[held].flatten())


# ------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2407_18121_b200 import binding as ec
    if op == "reserve":
        s["buffer"].copy_(s["before"])                      # the step before left it like this
        if own:
            ec.ec_paged_release(s["cache"], s["pages"])
            ec.ec_paged_reserve(s["cache"], s["pages"], s["counts"], s["starts"], s["granted"], s["slots"], s["positions"])
        else:
            _release_and_reserve(s)
        return {k: s[k] for k in ("lens", "seen", "held", "n_free", "free", "table", "starts", "granted", "slots", "positions")}
    if op == "rotary":
        if own:
            ec.ec_rotary(s["x"], s["out"], s["positions"], s["freqs"], c["rot"], c["pairs"] == "next", s["factor"], c["back"])
        else:
            s["out"].copy_(_turn(s["x"], s["positions"], s["freqs"], s["factor"], c["rot"], c["pairs"], c["back"]))
        return {"out": s["out"]}
    if op == "join":
        if own:
            ec.ec_paged_join(s["q"], s["q_out"], s["k"], s["v"], None, s["slots"], s["positions"], s["cache"], s["freqs"], c["rot"],
                             c["pairs"] == "next", s["factor"])
        else:
            _join(s)
        return {k: s[k] for k in ("q_out", "K", "V", "weight", "pos")}
    scale = 1.0 / math.sqrt(c["D"])
    if op == "attention":
        if own:
            ec.ec_paged_chunk_attention(s["q"], s["starts"], s["counts"], s["cache"], scale, s["out"], s["lse"], s["ws"])
        else:
            _attention(s)
        return {"out": s["out"], "lse": s["lse"]}
    s["weight"].copy_(s["before"])                          # as the step before left them
    if own:
        ec.ec_paged_chunk_weights(s["q"], s["lse"], s["starts"], s["counts"], s["cache"], scale, DECAY, s["ws"])
    else:
        _weights(s)
    return {"weight": s["weight"]}


# ------------------------------------------------------------------ the definition, in 64 bits

def _exact_pages(s):
    """Problem by problem on the host, as lists and a stack."""
    c = s["case"]
    N, ps = c["N"], c["page"]
    lens, seen, held, counts = (s[k].tolist() for k in ("lens", "seen", "held", "counts"))
    table, free, height = s["table"].cpu().clone(), s["free"].cpu().clone(), int(s["n_free"])
    for n in range(N):
        keep = min(held[n], -(-max(lens[n], 0) // ps))
        for p in range(keep, held[n]):
            free[height] = table[n, p]
            height += 1
        held[n] = keep
    starts, granted, slots, positions, top, refused = [0], [], [], [], height, False
    for n in range(N):
        cnt = max(counts[n], 0)
        fits = lens[n] >= 0 and lens[n] + cnt <= table.shape[1] * ps and starts[-1] + cnt <= s["tokens"]
        need = max(0, -(-(lens[n] + cnt) // ps) - held[n]) if fits and cnt else 0
        ok = fits and (need == 0 or (not refused and need <= height))
        refused = refused or (need > 0 and not ok)
        if ok:
            for _ in range(need):
                height -= 1
                table[n, held[n]] = free[height]
                held[n] += 1
        for t in range(cnt):
            row = lens[n] + t
            slots.append(int(table[n, row // ps]) * ps + row % ps if ok else -1)
            positions.append(seen[n] + t if ok else -1)
        starts.append(starts[-1] + cnt)
        granted.append(cnt if ok else 0)
        lens[n] += granted[-1]
        seen[n] += granted[-1]
    rest = s["tokens"] - len(slots)
    whole = dict(lens=lens, seen=seen, held=held, n_free=[height], starts=starts, granted=granted, slots=slots + [-1] * rest,
                 positions=positions + [-1] * rest)
    got = {k: torch.tensor(v, dtype=torch.int32, device="cuda") for k, v in whole.items()}
    return {**got, "free": free.cuda(), "table": table.cuda()}


def _exact_turn(x, positions, freqs, factor, rot, pairs, back):
    """As a product of complex numbers."""
    x = x.double()
    z = x[..., :rot]
    z = torch.complex(z[..., 0::2], z[..., 1::2]) if pairs == "next" else torch.complex(z[..., :rot // 2], z[..., rot // 2:])
    angle = positions.double()[..., None, None] * freqs
    z = z * torch.polar(torch.full_like(angle, factor), -angle if back else angle)
    z = torch.view_as_real(z).flatten(-2) if pairs == "next" else torch.cat([z.real, z.imag], -1)
    return torch.cat([z, x[..., rot:]], -1)


def exact(case, seed):
    was = own
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = was
    op = case["op"]
    if op == "reserve":
        return _exact_pages(s)
    if op == "rotary":
        return {"out": _exact_turn(s["x"], s["positions"], s["freqs"], s["factor"], case["rot"], case["pairs"], case["back"])}
    H, G, D, ps = (case[k] for k in ("H", "G", "D", "page"))
    if op == "join":
        how = (s["positions"], s["freqs"], s["factor"], case["rot"], case["pairs"], False)
        K, V = s["K"].double(), s["V"].double()
        weight, pos = s["weight"].double(), s["pos"].clone()
        page, place = s["slots"].long() // ps, s["slots"].long() % ps
        K[page, :, place], V[page, :, place] = _exact_turn(s["k"], *how), s["v"].double()
        weight[page, :, place] = 0.0
        pos[page, :, place] = s["positions"][:, None].expand(-1, H)
        return {"q_out": _exact_turn(s["q"], *how), "K": K, "V": V, "weight": weight, "pos": pos}
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    weight = s["weight"].double()
    for n, (count, length, start) in enumerate(zip(s["counts"].tolist(), s["lens"].tolist(), s["starts"].tolist())):
        if count == 0:
            continue
        pages = s["table"][n, :-(-length // ps)].long()
        row = torch.arange(length, device="cuda")
        limit = (length - count + torch.arange(count, device="cuda")).repeat_interleave(G)
        hidden = row[None] > limit[:, None]
        share = torch.pow(torch.tensor(DECAY, dtype=torch.float64, device="cuda"), (length - 1 - limit).double())
        for h in range(H):
            K = s["K"][pages, h].reshape(-1, D)[:length].double()
            V = s["V"][pages, h].reshape(-1, D)[:length].double()
            q = s["q"][start:start + count, h * G:(h + 1) * G].reshape(-1, D).double()
            for a in range(0, count * G, 8192):                                                 # a slab of query rows
                b = min(a + 8192, count * G)
                x = (q[a:b] @ K.T / D ** 0.5).masked_fill_(hidden[a:b], -math.inf)
                if op == "attention":
                    z = torch.logsumexp(x, -1)
                    o = torch.exp_(x.sub_(z[:, None])) @ V
                    at = torch.arange(a, b, device="cuda")
                    out[start + at // G, h * G + at % G], lse[start + at // G, h * G + at % G] = o, z
                else:
                    z = s["lse"][start:start + count, h * G:(h + 1) * G].reshape(-1)[a:b].double()
                    if a == 0:
                        weight[pages[row // ps], h, row % ps] *= DECAY ** count
                    weight[pages[row // ps], h, row % ps] += share[a:b] @ torch.exp_(x.sub_(z[:, None]))
    return {"out": out, "lse": lse} if op == "attention" else {"weight": weight}
