"""Plain 64-bit forms of the paged cache's operators, on the CPU, row by row as they are defined. Used by the tests only."""
import math

import numpy as np
import torch


class PagedMirror:
    """A paged cache and its host copy. `garbage` fills what no row occupies, to show that nothing reads or writes it."""

    def __init__(self, lens, H, D, page, cap, dtype=torch.bfloat16, rows="heads", seed=0, device="cuda", spare=2, G=1,
                 garbage=float("nan"), ranked=False):
        g = torch.Generator().manual_seed(seed)
        N, self.page = len(lens), page
        self.max_pages = -(-cap // page)
        n_pages = N * self.max_pages + spare
        self.table = torch.randperm(n_pages, generator=g)[:N * self.max_pages].view(N, self.max_pages).to(torch.int32)
        shape = (n_pages, H, page, D)
        K, V = (torch.full(shape, garbage, dtype=dtype) for _ in range(2))
        weight = torch.full(shape[:3], garbage)
        pos = torch.full(shape[:3], -7, dtype=torch.int32)
        for n, length in enumerate(lens):
            if length <= 0:
                continue
            p, s = self.where(n, length)
            K[p, :, s] = torch.randn(length, H, D, generator=g).to(dtype)
            V[p, :, s] = torch.randn(length, H, D, generator=g).to(dtype)
            if ranked:                       # weights further apart than a step can add, so that no decision hangs on a rounding
                weight[p, :, s] = torch.stack([torch.randperm(length, generator=g) for _ in range(H)], 1).float() * (G + 1.0)
            else:
                weight[p, :, s] = torch.rand(length, H, generator=g)
            pos[p, :, s] = torch.stack([torch.randperm(3 * length, generator=g)[:length] for _ in range(H)], 1).to(torch.int32)
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.seen = torch.where(self.lens >= 0, 3 * self.lens, self.lens)
        self.H, self.D, self.N, self.dtype = H, D, N, dtype
        self.K, self.V, self.weight, self.pos = K, V, weight, pos
        if device is not None:
            def up(t):
                if rows == "tokens":
                    return t.transpose(1, 2).contiguous().to(device).transpose(1, 2)
                return t.to(device)
            self.dev = dict(K=up(K), V=up(V), weight=weight.to(device), pos=pos.to(device), table=self.table.to(device),
                            lens=self.lens.to(device), seen=self.seen.to(device))
        self.weight = weight.double()        # the mirror gathers in 64 bits

    def where(self, n, upto):
        r = torch.arange(upto)
        return self.table[n].long()[r // self.page], r % self.page

    def cache(self, ec):
        d = self.dev
        state = torch.empty(ec.ec_paged_state_bytes(self.N), dtype=torch.uint8, device=d["K"].device)
        return ec.ec_paged_init(d["K"], d["V"], d["weight"], d["pos"], d["table"], d["lens"], d["seen"], state)

    # -------------------------------------------------------------- definitions
    def attention(self, q, k_new, v_new, scale, accumulate=False, decay=1.0, drop=()):
        """Returns out, lse, w_new (float64) and bounds: `mass` = sum p |v| per output, `dx` the largest error of a score
        that fp32 accumulation of its D products can make. `drop`: (n, row) pairs that count as absent."""
        N, H, D = self.N, self.H, self.D
        G = q.shape[1] // H
        out = torch.zeros(N, H, G, D, dtype=torch.float64)
        mass, lse = torch.zeros_like(out), torch.full((N, H, G), -math.inf, dtype=torch.float64)
        w_new, dx = torch.zeros(N, H, dtype=torch.float64), 0.0
        for n, length in enumerate(self.lens.tolist()):
            if length < 0:
                continue
            p_, s_ = self.where(n, length)
            keep = torch.tensor([(n, j) not in drop for j in range(length)], dtype=torch.bool)
            p_, s_ = p_[keep], s_[keep]
            K, V = self.K[p_, :, s_].double(), self.V[p_, :, s_].double()
            if k_new is not None:
                K, V = torch.cat([K, k_new[n][None].double()]), torch.cat([V, v_new[n][None].double()])
            if K.shape[0] == 0:
                continue
            qn = q[n].double().view(H, G, D)
            x = torch.einsum("hgd,lhd->hgl", qn, K) * scale
            fine = torch.where(torch.isfinite(x), torch.einsum("hgd,lhd->hgl", qn.abs(), K.abs()) * scale, torch.zeros_like(x))
            dx = max(dx, float(fine.max()) * D * 2.0 ** -23)
            m = x.amax(-1, keepdim=True)
            e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
            z = e.sum(-1, keepdim=True)
            p = torch.where(z == 0, torch.zeros_like(e), e / z)
            lse[n] = (torch.log(z) + m)[..., 0]
            out[n] = torch.einsum("hgl,lhd->hgd", p, V)
            mass[n] = torch.einsum("hgl,lhd->hgd", p, V.abs())
            w = p.sum(1)
            if k_new is not None:
                w_new[n] = w[:, -1]
                w = w[:, :-1]
            if accumulate:
                self.weight[p_, :, s_] = decay * self.weight[p_, :, s_] + w.T
        return (out.view(N, H * G, D), lse.view(N, H * G), w_new), mass.view(N, H * G, D), dx

    def append(self, K_new, V_new, w_new, pos_new, counts, T, fresh, budget, recent, sinks):
        for n, length in enumerate(self.lens.tolist()):
            if length < 0:
                continue
            had, before = (0, 0) if fresh else (length, int(self.seen[n]))
            cnt = T if counts is None else max(0, min(T, int(counts[n])))
            after, final = before + cnt, min(had + cnt, budget)
            p_, s_ = self.where(n, max(had, final))
            for h in range(self.H):
                w = [float(v) for v in self.weight[p_[:had], h, s_[:had]]]
                w += [0.0 if w_new is None else float(w_new[n, h, t]) for t in range(cnt)]
                at = [int(v) for v in self.pos[p_[:had], h, s_[:had]]]
                at += [before + t if pos_new is None else int(pos_new[n, h, t]) for t in range(cnt)]

                def key(j):
                    safe = at[j] < sinks or at[j] >= after - recent
                    nan = math.isnan(w[j])
                    return (0 if safe else 1, 0 if nan else 1, 0.0 if nan else -w[j], j)
                best = sorted(range(had + cnt), key=key)[:final]
                stay = {j for j in best if j < min(had, final)}
                holes = [j for j in range(final) if j not in stay]
                come = sorted(j for j in best if j not in stay)
                for pool, new in ((self.K, K_new), (self.V, V_new)):
                    rows = [pool[p_[j], h, s_[j]].clone() if j < had else new[n, h, j - had].clone() for j in come]
                    for dst, row in zip(holes, rows):
                        pool[p_[dst], h, s_[dst]] = row
                for dst, j in zip(holes, come):
                    self.weight[p_[dst], h, s_[dst]] = w[j]
                    self.pos[p_[dst], h, s_[dst]] = at[j]
            self.lens[n], self.seen[n] = final, after

    # -------------------------------------------------------------- comparisons
    def assert_same_rows(self, weight_atol=0.0, what=""):
        """K, V, pos, lens, seen bit for bit over the whole pool, weights within `weight_atol`."""
        d = self.dev

        def bits(t):
            return t.cpu().contiguous().view(torch.int16)
        assert torch.equal(d["lens"].cpu(), self.lens), what + ": lens"
        assert torch.equal(d["seen"].cpu(), self.seen), what + ": seen"
        assert torch.equal(d["pos"].cpu(), self.pos), what + ": pos"
        assert torch.equal(bits(d["K"]), bits(self.K)), what + ": K"
        assert torch.equal(bits(d["V"]), bits(self.V)), what + ": V"
        got, want = d["weight"].cpu().double().numpy(), self.weight.numpy()
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
        same = (got == want) | np.isnan(want)
        got, want = np.where(same, 0.0, got), np.where(same, 0.0, want)
        assert (same | (np.abs(got - want) <= weight_atol)).all(), \
            f"{what}: weight off by {np.nanmax(np.abs(got - want)):.3g}, allowed {weight_atol:.3g}"


def attention_bounds(ref, mass, dx, dtype, G):
    """Tolerances of (out, lse, weight-per-step). A probability is off by 2 dx (its own score and the normaliser) and by
    a few fp32 roundings of the exponential, its product and its sum (2^-19 in all); P and the result are each rounded
    once to the element type, by half a step relative to the value."""
    out, lse, _ = ref
    half = torch.finfo(dtype).eps / 2
    p_rel = 2 * dx + 2.0 ** -19
    tiny = torch.finfo(dtype).tiny * half * 2                 # results below the smallest normal number: absolute steps
    out_tol = half * out.abs() + (half + p_rel) * (1 + half) * mass + tiny * (1 + mass)
    if dtype == torch.float16:                                # P below fp16's normal range is rounded in absolute steps of 2^-24
        out_tol = out_tol + 2.0 ** -25 * mass.amax() * 64
    lse_tol = dx + 2.0 ** -21 * (1 + torch.where(torch.isfinite(lse), lse.abs(), torch.zeros_like(lse)))
    return out_tol, lse_tol, G * p_rel
