"""Plain 64-bit forms of the chunk operators, on the CPU, and how far the kernels may be off them. Used by the tests only.

Tolerances, element by element, from what the kernels round (half = half a step of the type, relative to the value):
  score        D exact products summed in fp32 by steps that may cut instead of round: off by D 2^-23 sum |q k|, times scale
  exponent     scale * log2(e), the scaled maximum and the scaled normaliser are rounded to fp32 and so is the exponent: 2^-22 of the
               largest of |x|, |lse|; the exponential itself 2^-17 (the polynomial's 6e-6)
  P for V      rounded once: half. fp16: a multiple of 2^-24 where 2^11 stands for the maximum, 2^-36 of the largest probability
  sums         a thread adds the columns of its row one pair after the other: rows / 2 + 64 roundings of 2^-24; products are added in fp32
               by steps that may cut: rows + 64 of 2^-23; parts of a split row are scaled and added: 300 of 2^-24 more
  result       rounded once
"""
import math

import torch

F64 = torch.float64


class ChunkExact:
    """Attention and weights of a chunk over a mirror whose lengths count the chunk's rows."""

    def __init__(self, m, q, starts, counts, scale, decay=1.0, lse=None, drop=()):
        """q [tokens, Hq, D]; lse: the normaliser that the weights start from (its own when None); drop: (n, row) pairs that are absent."""
        H, D, G = m.H, m.D, q.shape[1] // m.H
        half = torch.finfo(m.dtype).eps / 2
        T, Hq = q.shape[:2]
        self.out, self.out_tol = torch.zeros(T, Hq, D, dtype=F64), torch.zeros(T, Hq, D, dtype=F64)
        self.lse, self.lse_tol = torch.full((T, Hq), -math.inf, dtype=F64), torch.zeros(T, Hq, dtype=F64)
        self.owned = torch.zeros(T, dtype=torch.bool)
        self.weight, self.weight_tol = m.weight.clone(), torch.zeros_like(m.weight)
        for n, length in enumerate(m.lens.tolist()):
            cnt, start = int(counts[n]), int(starts[n])
            if cnt <= 0:
                continue
            self.owned[start:start + cnt] = True
            rows = max(length, 0)
            keep = torch.tensor([(n, j) not in drop for j in range(rows)], dtype=torch.bool)
            page, slot = m.where(n, rows)
            page, slot = page[keep], slot[keep]
            at = torch.arange(rows)[keep]
            K, V = m.K[page, :, slot].double(), m.V[page, :, slot].double()                     # [rows, H, D]
            qn = q[start:start + cnt].double().view(cnt, H, G, D)
            x = torch.einsum("thgd,lhd->thgl", qn, K) * scale
            ax = torch.einsum("thgd,lhd->thgl", qn.abs(), K.abs()) * scale
            sees = at[None] <= (rows - cnt + torch.arange(cnt))[:, None]                        # [cnt, rows]
            sees = sees[:, None, None].expand_as(x)
            x = x.masked_fill(~sees, -math.inf)
            mx = x.amax(-1, keepdim=True) if rows and len(at) else torch.full((cnt, H, G, 1), -math.inf, dtype=F64)
            base = torch.where(mx == -math.inf, torch.zeros_like(mx), mx)
            e = torch.exp(x - base)
            z = e.sum(-1, keepdim=True)
            p = torch.where(z == 0, torch.zeros_like(e), e / z)
            p_v = torch.where(sees, p, torch.zeros_like(p))
            lse_n = (torch.log(z) + base)[..., 0]
            fine = torch.where(sees & torch.isfinite(x), ax, torch.zeros_like(ax))
            big = fine.amax(-1) if len(at) else torch.zeros(cnt, H, G, dtype=F64)
            xs = torch.where(sees & torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1) if len(at) else big
            p_rel = 2 * D * 2.0 ** -23 * big + 2.0 ** -17 + 4 * xs * 2.0 ** -22 + (rows / 2 + 364) * 2.0 ** -24
            out = torch.einsum("thgl,lhd->thgd", p_v, torch.nan_to_num(V, nan=0.0, posinf=0.0, neginf=0.0))
            mass = torch.einsum("thgl,lhd->thgd", p_v, torch.nan_to_num(V, nan=0.0, posinf=0.0, neginf=0.0).abs())
            spoilt = torch.einsum("tl,lhd->thd", (at[None] <= (rows - cnt + torch.arange(cnt))[:, None]).double(),
                                  (~torch.isfinite(V)).double()) > 0
            out = torch.where(spoilt[:, :, None].expand_as(out), torch.full_like(out, math.nan), out)
            tol = half * out.abs() + (half + p_rel[..., None] + (rows + 64) * 2.0 ** -23) * mass * (1 + half)
            if m.dtype == torch.float16:
                top = p_v.amax(-1) if len(at) else torch.zeros(cnt, H, G, dtype=F64)
                tol = tol + 2.0 ** -36 * top[..., None] * torch.einsum("thgl,lhd->thgd", sees.double(), torch.nan_to_num(V, 0.0, 0.0, 0.0).abs())
            tol = tol + torch.finfo(m.dtype).tiny * half * 2
            sl = slice(start, start + cnt)
            self.out[sl], self.out_tol[sl] = out.reshape(cnt, Hq, D), tol.reshape(cnt, Hq, D)
            self.lse[sl] = lse_n.reshape(cnt, Hq)
            self.lse_tol[sl] = (p_rel + 2.0 ** -21 * (1 + torch.where(torch.isfinite(lse_n), lse_n.abs(), torch.zeros_like(lse_n)))).reshape(cnt, Hq)
            # weights
            zn = (lse_n if lse is None else lse[sl].double().view(cnt, H, G))[..., None]
            pw = torch.where(sees & (zn != -math.inf), torch.exp(x - zn), torch.zeros_like(x))
            share = decay ** (cnt - 1 - torch.arange(cnt, dtype=F64))
            gain = torch.einsum("t,thgl->lh", share, pw)
            zs = torch.where(torch.isfinite(zn), zn.abs(), torch.zeros_like(zn))[..., 0]
            w_rel = D * 2.0 ** -23 * big + 2.0 ** -17 + (xs + zs + cnt * abs(math.log(decay))) * 2.0 ** -21 + (cnt * G + 16) * 2.0 ** -24
            new = decay ** cnt * m.weight[page, :, slot] + gain
            self.weight[page, :, slot] = new
            self.weight_tol[page, :, slot] = torch.einsum("t,thgl->lh", share, pw * w_rel[..., None]) + 2.0 ** -22 * new.abs() + 2.0 ** -120

    def assert_out(self, got, lse=None, what=""):
        got = got.cpu().double()
        want = self.out[self.owned]
        mine = got[self.owned]
        assert torch.equal(torch.isnan(mine), torch.isnan(want)), what + ": NaN where there should be none, or the other way round"
        over = torch.nan_to_num((mine - want).abs() - self.out_tol[self.owned], nan=-1.0)
        assert (over <= 0).all(), f"{what} out: {int((over > 0).sum())} elements over, the worst by {float(over.max()):.3g}"
        if lse is not None:
            g, w = lse.cpu().double()[self.owned], self.lse[self.owned]
            empty = torch.isinf(w)
            assert torch.equal(torch.isinf(g) & (g < 0), empty), what + " lse: empty rows"
            assert ((g - w).abs()[~empty] <= self.lse_tol[self.owned][~empty]).all(), what + " lse"

    def assert_weights(self, weight, what=""):
        got, took = weight.cpu().double(), self.weight_tol > 0
        over = ((got - self.weight).abs() - self.weight_tol)[took]
        assert (over <= 0).all(), f"{what} weights: {int((~(over <= 0)).sum())} over, the worst by {float(over.max()):.3g}"
        same = (got == self.weight) | (torch.isnan(got) & torch.isnan(self.weight))
        assert same[~took].all(), what + ": weights of rows that take no part"


def rotary(x, positions, freqs, factor, rot, interleaved, inverse=False):
    """x [..., heads, D] in 64 bits, positions [...]."""
    x = x.double().clone()
    # the angle's turns are taken out exactly: positions and frequencies are what they are
    angle = torch.remainder(positions.double()[..., None, None] * freqs.double(), 2 * math.pi)
    c, s = torch.cos(angle) * factor, torch.sin(angle) * factor * (-1 if inverse else 1)
    a, b = (x[..., 0:rot:2].clone(), x[..., 1:rot:2].clone()) if interleaved else (x[..., :rot // 2].clone(), x[..., rot // 2:rot].clone())
    p, q = a * c - b * s, a * s + b * c
    if interleaved:
        x[..., 0:rot:2], x[..., 1:rot:2] = p, q
    else:
        x[..., :rot // 2], x[..., rot // 2:rot] = p, q
    return x


class PoolModel:
    """Pages of a pool as lists and a stack."""

    def __init__(self, lens, seen, held, table, free, page):
        self.lens, self.seen, self.held, self.page = list(lens), list(seen), list(held), page
        self.table, self.free = [list(r) for r in table], list(free)

    def release(self):
        for n in range(len(self.lens)):
            keep = min(self.held[n], -(-max(self.lens[n], 0) // self.page))
            self.free += self.table[n][keep:self.held[n]]
            self.held[n] = keep

    def reserve(self, counts, tokens, advance=True, limit=0):
        starts, granted, slots, positions, asked, full = [0], [], [], [], 0, False
        height = len(self.free)
        total = 0
        for n, cnt in enumerate(max(c, 0) for c in counts):
            rows = self.lens[n] + cnt
            if not advance and limit:
                rows = min(rows, max(limit, self.lens[n]))
            total += cnt
            fits = self.lens[n] >= 0 and rows <= len(self.table[n]) * self.page and (not advance or total <= tokens)
            need = max(0, -(-rows // self.page) - self.held[n]) if fits and cnt else 0
            asked += need
            ok = fits and (need == 0 or asked <= height)
            if ok:
                for _ in range(need):
                    self.table[n][self.held[n]] = self.free.pop()
                    self.held[n] += 1
            if advance:
                for t in range(cnt):
                    row = self.lens[n] + t
                    slots.append(self.table[n][row // self.page] * self.page + row % self.page if ok else -1)
                    positions.append(self.seen[n] + t if ok else -1)
                if ok:
                    self.lens[n] += cnt
                    self.seen[n] += cnt
            starts.append(min(starts[-1] + cnt, tokens))
            granted.append(cnt if ok else 0)
        pad = [-1] * max(0, tokens - len(slots))
        return starts, granted, (slots + pad)[:tokens], (positions + pad)[:tokens]
