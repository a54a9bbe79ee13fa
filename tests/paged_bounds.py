"""Tolerances of the paged attention, element by element, from what the kernel rounds. Used by the tests only.

  score        D exact products, summed in fp32 by steps that may cut instead of round: off by D 2^-23 sum |q k|
  probability  twice the largest of those of its head (its own score and the normaliser), the exponential's argument and result and
               the factors that join parts (2^-19 in all), and the sum of the normaliser: a lane adds one of 64 rows at most, then
               lanes, warps and parts are added
  P for V      the sum of two parts. bf16: each rounded, which leaves half^2 of P. fp16: two parts that are multiples of 2^-24 where 2^11
               stands for the maximum, which leaves 2^-36 of the maximum's, as long as that is no more than 2^-14 of P; else, as
               well as beside it, parts of 11 bits with fp32's exponents, cut, which leaves 2^-20 of P
  product      fp32 sums by steps that may cut: two per row of the warp's (a quarter of the rows at most), then warps and parts
  result       rounded once to the element type

`half` is half a step of the type relative to the value, finfo.eps / 2."""
import math

import torch


class Exact:
    """64-bit attention of one new token per problem over a mirror of the cache, and how far the kernel may be off it."""

    def __init__(self, m, q, k_new, v_new, scale, decay=1.0):
        N, H, D, G = m.N, m.H, m.D, q.shape[1] // m.H
        half = torch.finfo(m.dtype).eps / 2
        f64 = torch.float64
        self.out, self.lse = torch.zeros(N, H, G, D, dtype=f64), torch.full((N, H, G), -math.inf, dtype=f64)
        self.out_tol, self.lse_tol = torch.zeros_like(self.out), torch.zeros_like(self.lse)
        self.weight, self.weight_tol = m.weight.clone(), torch.zeros_like(m.weight)
        self.w_new, self.w_new_tol = torch.zeros(N, H, dtype=f64), torch.zeros(N, H, dtype=f64)
        self.gain = torch.zeros_like(m.weight)
        self.parts = []                      # (n, p, V) of every problem that has rows
        for n, length in enumerate(m.lens.tolist()):
            if length < 0 or length + (k_new is not None) == 0:
                continue
            page, slot = m.where(n, length)
            K, V = m.K[page, :, slot].double(), m.V[page, :, slot].double()
            if k_new is not None:
                K, V = torch.cat([K, k_new[n][None].double()]), torch.cat([V, v_new[n][None].double()])
            rows = K.shape[0]
            qn = q[n].double().view(H, G, D)
            x = torch.einsum("hgd,lhd->hgl", qn, K) * scale
            dx = (torch.einsum("hgd,lhd->hgl", qn.abs(), K.abs()) * scale * D * 2.0 ** -23).amax(-1)          # [H, G]
            p = torch.softmax(x, -1)
            parts = rows / 64 + 2
            p_rel = 2 * dx + 2.0 ** -19 + (rows / 64 + 16 + parts) * 2.0 ** -24
            sums = (2 * (rows / 4 + 32) + 16 + parts) * 2.0 ** -23
            mass = torch.einsum("hgl,lhd->hgd", p, V.abs())
            self.out[n] = torch.einsum("hgl,lhd->hgd", p, V)
            p_off = half ** 2 * p
            if m.dtype == torch.float16:
                p_off = 2.0 ** -20 * p + torch.minimum(2.0 ** -36 * p.amax(-1, keepdim=True), 2.0 ** -14 * p)
            before = torch.einsum("hgl,lhd->hgd", p_off, V.abs()) + (sums + p_rel[..., None]) * mass
            tiny = torch.finfo(m.dtype).tiny * half * 2                   # results below the smallest normal number: absolute steps
            self.out_tol[n] = (half * self.out[n].abs() + before) * (1 + 2 * half) + tiny
            self.lse[n] = torch.logsumexp(x, -1)
            self.lse_tol[n] = p_rel + 2.0 ** -21 * (1 + self.lse[n].abs())
            w, w_tol = p.sum(1), (p * p_rel[..., None]).sum(1)                                                # [H, rows]
            if k_new is not None:
                self.w_new[n], self.w_new_tol[n] = w[:, -1], w_tol[:, -1] + G * 2.0 ** -24 * w[:, -1]
                w, w_tol = w[:, :-1], w_tol[:, :-1]
            new = decay * m.weight[page, :, slot] + w.T
            self.weight[page, :, slot] = new
            self.gain[page, :, slot] = w.T
            self.weight_tol[page, :, slot] = w_tol.T + G * 2.0 ** -24 * w.T + 2.0 ** -24 * new.abs() * (1 + 2.0 ** -20)
            self.parts.append((n, p, V))

    def with_rounded_p(self, dtype):
        """The outputs (not rounded) of a kernel that rounds P once, to `dtype`, relative to the largest of its head."""
        out = torch.zeros_like(self.out)
        for n, p, V in self.parts:
            top = p.amax(-1, keepdim=True)
            out[n] = torch.einsum("hgl,lhd->hgd", (p / top).to(dtype).double() * top, V)
        return out

    def assert_out(self, got, what=""):
        over = (got.cpu().double().view_as(self.out) - self.out).abs() - self.out_tol
        assert (over <= 0).all(), f"{what} out: {int((~(over <= 0)).sum())} elements over, the worst by {float(over.max()):.3g}"

    def assert_lse(self, got, what=""):
        got, empty = got.cpu().double().view_as(self.lse), torch.isinf(self.lse)
        assert torch.equal(torch.isinf(got), empty)
        assert ((got - self.lse).abs()[~empty] <= self.lse_tol[~empty]).all(), what + " lse"

    def assert_weights(self, weight, w_new=None, what=""):
        got, held = weight.cpu().double(), self.weight_tol > 0
        over = ((got - self.weight).abs() - self.weight_tol)[held]
        assert (over <= 0).all(), f"{what} weights: {int((~(over <= 0)).sum())} over, the worst by {float(over.max()):.3g}"
        same = (got == self.weight) | (torch.isnan(got) & torch.isnan(self.weight))
        assert same[~held].all(), what + " weights of rows that take no part"
        if w_new is not None:
            assert ((w_new.cpu().double() - self.w_new).abs() <= self.w_new_tol).all(), what + " w_new"
