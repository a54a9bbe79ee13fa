"""Operators of the paged cache, with their plain forms.

Three calls work on a pool of pages that holds the key / value rows of N independent problems (sequence x layer
folded), H key / value heads each, together with the attention weight every row has gathered so far and the token
position it came from:

  attention  one new token per problem over its cached rows and its own row, Hq = H * G query heads, the probability
             that each row receives added to its weight:
                 out = softmax(scale * q [K; k_new]^T) [V; v_new],   weight <- decay * weight + sum over the G heads of p
  append     T new rows per problem join the cached ones; when a problem then has more than `budget` rows, every head
             keeps the `budget` rows of largest weight (equal weights: the lower index, cached rows before new ones),
             with the first `sinks` and the newest `recent` token positions always kept. Kept rows stay where they
             are; the holes below the new length are filled, in ascending order, by the kept rows from behind it
             (cached ones first, then the new ones in order)
  step       one generation step: attention with the weights gathered, then append of the step's own row

A problem whose length is negative is an empty place of a padded batch: its output is zero and nothing of it changes.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
RECENT, SINKS = 16, 4
KEEP = 1.0                                  # decay of the gathered weights: a plain sum


def listed():
    return [
        # one user, a question just begun: nothing but latency
        dict(name="attention short", op="attention", N=1, H=8, G=4, D=128, L=37, ragged=False, page=16, dtype="bf16", rows="heads", weights=False),
        # a serving batch at all stages of its answers, grouped query heads, rows of a page shared by the heads side by side
        dict(name="attention ragged batch", op="attention", N=32, H=8, G=4, D=128, L=8192, ragged=True, page=64, dtype="bf16", rows="tokens", weights=False),
        # one very long context: all parallelism comes from its length
        dict(name="attention long", op="attention", N=1, H=8, G=8, D=128, L=131071, ragged=False, page=64, dtype="bf16", rows="heads", weights=False),
        # a 7B-shaped model's 32 layers with one head group per head, weights gathered, prompt of 640 rows
        dict(name="attention weights 640", op="attention", N=32, H=32, G=1, D=128, L=640, ragged=False, page=16, dtype="bf16", rows="heads", weights=True),
        # odd group, odd pages, smaller heads, half precision, ragged
        dict(name="attention weights odd", op="attention", N=24, H=5, G=7, D=64, L=2047, ragged=True, page=24, dtype="fp16", rows="heads", weights=True),
        # four layers of a batch of four at 8192 rows: bandwidth
        dict(name="attention weights 8192", op="attention", N=16, H=32, G=1, D=128, L=8192, ragged=False, page=128, dtype="bf16", rows="heads", weights=True),
        # the step's row into a cache that is at its budget, 7B shapes
        dict(name="append token", op="append", N=32, H=32, D=128, L=320, T=1, fresh=False, budget=320, ragged=False, page=16, dtype="bf16", rows="heads"),
        # a whole prompt into empty pages at keep ratio 0.5, 7B shapes
        dict(name="append prompt 640", op="append", N=32, H=32, D=128, L=0, T=640, fresh=True, budget=320, ragged=False, page=16, dtype="bf16", rows="heads"),
        # two long prompts of different lengths, few heads: all parallelism comes from the length
        dict(name="append prompt 16384", op="append", N=2, H=8, D=64, L=0, T=16384, fresh=True, budget=4096, ragged=True, page=64, dtype="fp16", rows="heads"),
        # a further instruction on top of full caches
        dict(name="append instruction", op="append", N=32, H=8, D=128, L=2048, T=64, fresh=False, budget=2048, ragged=True, page=64, dtype="bf16", rows="tokens"),
        # whole steps: 7B shapes at budget 320, and a grouped-head batch with empty places at budget 2048
        dict(name="step 320", op="step", N=32, H=32, G=1, D=128, L=320, budget=320, ragged=False, page=16, dtype="bf16", rows="heads"),
        dict(name="step 2048", op="step", N=64, H=8, G=4, D=128, L=2048, budget=2048, ragged=True, page=64, dtype="bf16", rows="heads"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "append", "step"])
    c = dict(op=op, H=rng.choice([1, 2, 4, 5, 8, 16, 32, 40]), D=rng.choice([64, 128]), page=rng.choice([1, 8, 16, 24, 64, 100, 128]),
             dtype=rng.choice(["bf16", "fp16"]), rows=rng.choice(["heads", "tokens"]), ragged=rng.random() < 0.5)
    c["N"] = _log(rng, 1, 64)
    most = (1 << 29) // (c["N"] * c["H"] * c["D"])                      # rows of the largest listed case
    if op == "attention":
        c.update(G=rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16, 20]), weights=rng.random() < 0.5)
        c["L"] = _log(rng, 1, min(131072, most // max(1, c["G"] // 4)))
    elif op == "append":
        c["fresh"] = rng.random() < 0.5
        most = min(16384, most // 16)
        if c["fresh"]:
            c.update(L=0, T=_log(rng, 1, most))
            c["budget"] = max(RECENT + SINKS, _log(rng, 1, c["T"]))
        else:
            c.update(L=max(2 * (RECENT + SINKS), _log(rng, 1, most)))
            c["budget"] = c["L"]
            c["T"] = min(_log(rng, 1, 256), c["L"] // 2)
    else:
        c.update(G=rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]))
        c["L"] = c["budget"] = max(2 * (RECENT + SINKS), _log(rng, 1, min(8192, most // 8)))
    return c


# ------------------------------------------------------------------ shapes that a case fixes

def _lens(case):
    """Cached rows of every problem; part of the case, not of its seed."""
    N, L = case["N"], case["L"]
    lens = [L] * N
    if case["ragged"] and case["op"] == "attention":
        r = random.Random(7 * N + L)
        lens = [L] + [_log(r, 1, L) for _ in range(N - 1)]
        if N > 3:
            lens[2], lens[3] = 0, -1                # a problem with nothing cached yet, and an empty place
    elif case["ragged"] and case["op"] == "step" and N > 3:
        lens[1::4] = [-1] * len(lens[1::4])         # a quarter of the places is empty
    return lens


def _counts(case):
    """New rows of every problem in an append."""
    N, T = case["N"], case["T"]
    if not case["ragged"]:
        return [T] * N
    r = random.Random(11 * N + T)
    got = [T] + [_log(r, 1, T) for _ in range(N - 1)]
    if N > 3:
        got[1] = 0
    return got


def _recent(case):
    return case["T"] if case["op"] == "append" and not case["fresh"] else RECENT


def _budget(case):
    return case["budget"]


def work(case):
    H, D = case["H"], case["D"]
    lens = _lens(case)
    row = 2 * D * 2                                                     # bytes of a K row and a V row
    nbytes = flops = 0
    if case["op"] != "append":
        G = case["G"]
        live = [x for x in lens if x >= 0]
        rows = sum(live)
        nbytes += rows * H * row + len(live) * H * row + 2 * case["N"] * H * G * D * 2 + 4 * sum(-(-x // case["page"]) for x in live)
        flops += 4 * H * G * D * (rows + len(live))
        if case["op"] == "step" or case["weights"]:
            nbytes += 8 * rows * H
    if case["op"] != "attention":
        counts = _counts(case) if case["op"] == "append" else [1 if x >= 0 else 0 for x in lens]
        cached = sum(x for x in lens if x > 0)
        kept = sum(min(c, case["budget"]) for c in counts)
        nbytes += cached * H * 8 + sum(counts) * H * 4 + kept * H * (2 * row + 8)
        flops += (cached + sum(counts)) * H
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    op, N, H, D, L, ps = (case[k] for k in ("op", "N", "H", "D", "L", "page"))
    dt = DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    most = L + 1 if op == "attention" else case["budget"]
    max_pages = -(-most // ps)
    n_pages = N * max_pages + 3
    s = {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    # heavy hitters: every key has a share of one direction that all queries of its head look along
    u = torch.randn(H, D, generator=g, device="cuda")
    u = u / u.norm(dim=-1, keepdim=True)

    def pool():
        if case["rows"] == "heads":
            return normal(n_pages, H, ps, D)
        return normal(n_pages, ps, H, D).permute(0, 2, 1, 3)
    s["K"], s["V"] = pool(), pool()
    s["K"].add_((1.5 * torch.randn(n_pages, H, ps, 1, generator=g, device="cuda").abs()).to(dt) * u.to(dt)[None, :, None, :])
    s["table"] = torch.randperm(n_pages, generator=g, device="cuda")[:N * max_pages].view(N, max_pages).to(torch.int32)
    s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    s["seen"] = torch.where(s["lens"] >= 0, 4 * s["lens"] + 16, s["lens"])
    # history of the rows: weights that lie apart by at least what one step can add, so that the row that leaves does not
    # hang on the last bit of a probability; positions in steps of three with the newest rows at the end
    cap = max_pages * ps
    i = torch.arange(cap, device="cuda")
    lens = s["lens"].clamp(min=0)
    at = torch.where(i[None] >= (lens - _recent(case))[:, None], s["seen"][:, None] - lens[:, None] + i[None], 3 * i[None])
    rank = torch.rand(N, H, cap, generator=g, device="cuda").argsort(-1) + 1
    s["weight"] = torch.rand(n_pages, H, ps, generator=g, device="cuda")
    s["pos"] = torch.full((n_pages, H, ps), -1, dtype=torch.int32, device="cuda")
    page, slot = s["table"].long()[:, i // ps], (i % ps)[None].expand(N, cap)
    s["weight"][page, :, slot] = rank.transpose(1, 2).float() * case.get("G", 1)
    s["pos"][page, :, slot] = at[:, :, None].expand(N, cap, H).to(torch.int32)

    if op != "append":
        Hq = H * case["G"]
        s["q"] = normal(N, Hq, D) + (math.sqrt(D) * u).to(dt).repeat_interleave(case["G"], 0)
        s["k_new"], s["v_new"] = normal(N, H, D), normal(N, H, D)
        s["out"] = torch.empty(N, Hq, D, dtype=dt, device="cuda")
        s["lse"] = torch.empty(N, Hq, device="cuda")
        s["w_new"] = torch.empty(N, H, device="cuda")
    if op == "append":
        T = case["T"]
        s["k_new"], s["v_new"] = normal(N, H, T, D), normal(N, H, T, D)
        # column sums of a prompt's attention: heavy-tailed, many of them equal at the low end
        w = torch.exp(1.5 * torch.randn(N, H, T, generator=g, device="cuda"))
        s["w_new"] = torch.where(w < 0.1, torch.zeros_like(w), w)
        s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if own:
        from paper_2407_18121_b200 import binding as ec
        state = torch.empty(ec.ec_paged_state_bytes(N), dtype=torch.uint8, device="cuda")
        s["cache"] = ec.ec_paged_init(s["K"], s["V"], s["weight"], s["pos"], s["table"], s["lens"], s["seen"], state)
        if op == "attention":
            need = ec.ec_paged_attention_workspace(s["cache"], H * case["G"], case["weights"])
        elif op == "append":
            need = ec.ec_paged_append_workspace(s["cache"], case["T"], case["budget"])
        else:
            need = ec.ec_paged_step_workspace(s["cache"], H * case["G"], case["budget"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms

def _rows(s, upto):
    """(page, slot) of the first `upto` rows of every problem, each [N, upto]."""
    ps = s["case"]["page"]
    i = torch.arange(upto, device="cuda")
    return s["table"].long()[:, i // ps], (i % ps)[None].expand(s["table"].shape[0], upto)


def _attention(s, gather):
    c = s["case"]
    N, H, G, D, L = (c[k] for k in ("N", "H", "G", "D", "L"))
    page, slot = _rows(s, L)
    K = torch.cat([s["K"][page, :, slot], s["k_new"][:, None]], 1).float().transpose(1, 2)      # [N, H, L + 1, D]
    V = torch.cat([s["V"][page, :, slot], s["v_new"][:, None]], 1).float().transpose(1, 2)
    q = s["q"].float().view(N, H, G, D)
    there = torch.arange(L + 1, device="cuda")[None] < s["lens"][:, None]
    there[:, L] = s["lens"] >= 0                                                                # the token's own row
    x = (q @ K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    x = x.masked_fill(~there[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    p = e / torch.where(z == 0, torch.ones_like(z), z)
    V = V.masked_fill(~there[:, None, :, None], 0.0)
    s["out"].copy_((p @ V).view(N, H * G, D))
    s["lse"].copy_((torch.log(z) + m).view(N, H * G))
    if gather:
        w = p.sum(2)                                                                            # over the group: [N, H, L + 1]
        old = s["weight"][page, :, slot]                                                        # [N, L, H]
        s["weight"][page, :, slot] = torch.where(there[:, :L, None], KEEP * old + w[:, :, :L].transpose(1, 2), old)
        s["w_new"].copy_(w[:, :, L])


def _append(s, T, counts, fresh):
    """K, V, w: [N, H, T(, D)] of the new rows; the cache is changed in place."""
    c = s["case"]
    N, H, D, L, B = c["N"], c["H"], c["D"], c["L"], c["budget"]
    live = s["lens"] >= 0
    had = torch.zeros_like(s["lens"]) if fresh else s["lens"].clamp(min=0)
    cnt = torch.where(live, counts if counts is not None else torch.full_like(had, T), torch.zeros_like(had))
    seen = torch.zeros_like(s["seen"]) if fresh else s["seen"].clamp(min=0)
    F = torch.minimum(had + cnt, torch.full_like(had, B))
    Kn, Vn, wn = s["k_new"].view(N, H, T, D), s["v_new"].view(N, H, T, D), s["w_new"].view(N, H, T)
    S = max(L, B)                                                       # slots looked at
    page, slot = _rows(s, B)

    def cached(pool):
        x = pool[page, :, slot].transpose(1, 2)                         # [N, H, B, ...]
        return x
    t = torch.arange(T, device="cuda")
    i = torch.arange(B, device="cuda")
    pos = torch.cat([cached(s["pos"]), (seen[:, None] + t).to(torch.int32)[:, None].expand(N, H, T)], 2)
    wt = torch.cat([cached(s["weight"]), wn], 2)
    there = torch.cat([i[None] < had[:, None], t[None] < cnt[:, None]], 1)[:, None].expand(N, H, B + T)
    total = (seen + cnt)[:, None, None]
    safe = there & ((pos < SINKS) | (pos >= total - _recent(c)))
    tier = torch.where(safe, 2, torch.where(there, 1, 0))
    order = wt.argsort(dim=-1, descending=True, stable=True)
    order = order.gather(-1, tier.gather(-1, order).argsort(dim=-1, descending=True, stable=True))
    rank = torch.empty_like(order).scatter_(-1, order, torch.arange(B + T, device="cuda").expand(N, H, B + T))
    kept = there & (rank < F[:, None, None])
    index = torch.arange(B + T, device="cuda")
    hole = (i < F[:, None])[:, None] & ~kept[:, :, :B]
    mover = kept & ((index >= B) | (index >= F[:, None]))[:, None].expand(N, H, B + T)
    # the k-th hole takes the k-th mover
    movers = torch.zeros(N, H, B + T + 1, dtype=torch.long, device="cuda")
    movers.scatter_(2, torch.where(mover, mover.cumsum(-1) - 1, B + T), index.expand(N, H, B + T))
    src = torch.where(hole, movers.gather(2, hole.cumsum(-1).clamp(min=1) - 1), i)              # [N, H, B]
    for pool, new in ((s["K"], Kn), (s["V"], Vn)):
        rows = torch.cat([cached(pool), new], 2)
        pool[page, :, slot] = rows.gather(2, src[..., None].expand(N, H, B, D)).transpose(1, 2)
    s["weight"][page, :, slot] = wt.gather(2, src).transpose(1, 2)
    s["pos"][page, :, slot] = pos.gather(2, src).transpose(1, 2)
    s["lens"].copy_(torch.where(live, F, s["lens"]))
    s["seen"].copy_(torch.where(live, seen + cnt, s["seen"]))


# ------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    scale = 1.0 / math.sqrt(c["D"])
    if c["op"] == "attention":
        if own:
            from paper_2407_18121_b200 import binding as ec
            ec.ec_paged_attention(s["q"], s["k_new"], s["v_new"], s["cache"], scale, c["weights"], KEEP, s["out"], s["lse"],
                                  s["w_new"] if c["weights"] else None, s["ws"])
        else:
            _attention(s, c["weights"])
        got = {"out": s["out"], "lse": s["lse"]}
        if c["weights"]:
            got.update(weight=s["weight"], w_new=s["w_new"])
        return got
    if c["op"] == "append":
        if own:
            from paper_2407_18121_b200 import binding as ec
            ec.ec_paged_append(s["k_new"], s["v_new"], s["w_new"], None, s["counts"], s["cache"], c["fresh"], c["budget"],
                               _recent(c), SINKS, s["ws"])
        else:
            _append(s, c["T"], s["counts"], c["fresh"])
        return {k: s[k] for k in ("K", "V", "weight", "pos", "lens", "seen")}
    if own:
        from paper_2407_18121_b200 import binding as ec
        ec.ec_paged_decode_step(s["q"], s["k_new"], s["v_new"], s["cache"], scale, KEEP, c["budget"], RECENT, SINKS, s["out"],
                                s["lse"], s["ws"])
    else:
        _attention(s, True)
        _append(s, 1, None, False)
    return {k: s[k] for k in ("out", "lse", "K", "V", "weight", "pos", "lens", "seen")}


# ------------------------------------------------------------------ the definition, in 64 bits

def _exact_attention(s, gather):
    """Problem by problem; returns out, lse and (gather) changes s['weight'] (float64) and fills s['w_new']."""
    c = s["case"]
    N, H, G, D, ps = (c[k] for k in ("N", "H", "G", "D", "page"))
    out = torch.zeros(N, H, G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((N, H, G), -math.inf, dtype=torch.float64, device="cuda")
    s["w_new"] = torch.zeros(N, H, dtype=torch.float64, device="cuda")
    for n, length in enumerate(s["lens"].tolist()):
        if length < 0:
            continue
        pages = s["table"][n, :-(-length // ps)].long()

        def dense(pool, own_row):
            rows = pool[pages].transpose(1, 2).reshape(-1, H, D)[:length]
            return torch.cat([rows, own_row[None]]).double()
        K, V = dense(s["K"], s["k_new"][n]), dense(s["V"], s["v_new"][n])
        x = torch.einsum("hgd,lhd->hgl", s["q"][n].double().view(H, G, D), K) / D ** 0.5
        lse[n] = torch.logsumexp(x, -1)
        p = torch.softmax(x, -1)
        out[n] = torch.einsum("hgl,lhd->hgd", p, V)
        if gather:
            w = p.sum(1)                                                # [H, length + 1]
            s["w_new"][n] = w[:, length]
            r = torch.arange(length, device="cuda")
            s["weight"][pages[r // ps], :, r % ps] = KEEP * s["weight"][pages[r // ps], :, r % ps] + w[:, :length].T
    return out.view(N, H * G, D), lse.view(N, H * G)


def _exact_append(s, T, counts, fresh):
    """Unit by unit on the host: which row goes where; the rows themselves are copied on the device."""
    c = s["case"]
    N, H, B, ps = c["N"], c["H"], c["budget"], c["page"]
    table, lens, seen = s["table"].cpu().numpy(), s["lens"].cpu().numpy().copy(), s["seen"].cpu().numpy().copy()
    weight, pos = s["weight"].cpu().numpy().astype(np.float64), s["pos"].cpu().numpy().copy()
    new_w = s["w_new"].view(N, H, T).cpu().numpy().astype(np.float64)
    from_slot, to_slot, from_new, to_new = [], [], [], []               # (page, head, slot) triples and (n, h, t)
    for n in range(N):
        if lens[n] < 0:
            continue
        had, before = (0, 0) if fresh else (int(lens[n]), int(seen[n]))
        cnt = T if counts is None else int(counts[n])
        after, final = before + cnt, min(had + cnt, B)
        pg, sl = table[n][np.arange(max(had, final)) // ps], np.arange(max(had, final)) % ps
        for h in range(H):
            w = np.concatenate([weight[pg[:had], h, sl[:had]], new_w[n, h, :cnt]])
            at = np.concatenate([pos[pg[:had], h, sl[:had]], before + np.arange(cnt)])
            must = (at < SINKS) | (at >= after - _recent(c))
            best = sorted(range(had + cnt), key=lambda j: (not must[j], -w[j], j))[:final]
            stay = {j for j in best if j < min(had, final)}
            holes = [j for j in range(final) if j not in stay]
            come = sorted(j for j in best if j not in stay)
            for dst, j in zip(holes, come):
                weight[pg[dst], h, sl[dst]], pos[pg[dst], h, sl[dst]] = w[j], at[j]
                if j < had:
                    from_slot.append((pg[j], h, sl[j]))
                    to_slot.append((pg[dst], h, sl[dst]))
                else:
                    from_new.append((n, h, j - had))
                    to_new.append((pg[dst], h, sl[dst]))
        lens[n], seen[n] = final, after

    def at3(v):
        a = torch.tensor(np.array(v, dtype=np.int64).reshape(-1, 3), device="cuda")
        return a[:, 0], a[:, 1], a[:, 2]
    for pool, new in ((s["K"], s["k_new"]), (s["V"], s["v_new"])):
        moved = pool[at3(from_slot)]
        pool[at3(to_new)] = new.view(N, H, T, -1)[at3(from_new)]
        pool[at3(to_slot)] = moved
    return weight, pos, lens, seen


def exact(case, seed):
    was = own
    globals()["own"] = False
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = was
    got = {}
    if case["op"] != "append":
        gather = case["op"] == "step" or case["weights"]
        s["weight"] = s["weight"].double()
        got["out"], got["lse"] = _exact_attention(s, gather)
        if gather:
            got["weight"] = s["weight"]
            if case["op"] == "attention":
                got["w_new"] = s["w_new"]
    if case["op"] != "attention":
        T = case["T"] if case["op"] == "append" else 1
        if case["N"] * case["H"] * (case["L"] + T) > 4_000_000:         # the host's sorting would take too long
            return None
        counts = s["counts"].cpu().numpy() if case["op"] == "append" and s["counts"] is not None else None
        got["weight"], got["pos"], got["lens"], got["seen"] = _exact_append(s, T, counts, case.get("fresh", False))
        got["K"], got["V"] = s["K"], s["V"]
    return got
