"""Angles of rotary positions, against whole-number arithmetic of 256 bits."""
import math

import pytest
import torch

from paper_2407_18121_b200 import binding as ec
from test_paged_gpu import HF

pytestmark = pytest.mark.gpu
BITS = 256


def two_pi():
    """2 pi * 2^BITS, by 16 atan(1/5) - 4 atan(1/239)."""
    one = 1 << (BITS + 64)

    def atan_of(n):
        term, total, k = one // n, 0, 0
        while term:
            total += (term if k % 2 == 0 else -term) // (2 * k + 1)
            term //= n * n
            k += 1
        return total
    return 2 * (16 * atan_of(5) - 4 * atan_of(239)) >> 64


@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_at_the_ends_of_the_positions_range(interleaved):
    """Every pair is (1, 0), so that it becomes factor * (cos, sin). An angle is off by 2^-24 of a half turn and by 2^-52 of itself (freq / 2 pi
    in 64 bits: the product rounds by 2^-53, the constant by 2^-53.8), sine, cosine and the product with the factor by 2^-21 of
    themselves, and the result is rounded once: where a sine is small, that shows the angle."""
    freqs = [1.0, 0.999, 0.1, 3.7, 50.0, 123.4, 1000.0, 1e-4]
    rot, factor, turn = 16, 1024.0, two_pi()
    assert abs(turn / (1 << BITS) - 2 * math.pi) < 1e-15
    g = torch.Generator().manual_seed(1)
    n = 20000
    pos = torch.cat([(1 << 31) - 1 - torch.randint(0, 1 << 24, (n,), generator=g), -(1 << 31) + torch.randint(0, 1 << 24, (n,), generator=g),
                     torch.randint(-4, 5, (8,), generator=g)]).to(torch.int32)
    x = torch.zeros(1, len(pos), 1, 64, dtype=HF)
    x[..., slice(0, rot, 2) if interleaved else slice(0, rot // 2)] = 1.0
    out = torch.empty_like(x, device="cuda")
    ec.ec_rotary(x.cuda(), out, pos.cuda(), torch.tensor(freqs, dtype=torch.float64).cuda(), rot, interleaved, factor)
    got = out.cpu().double()[0, :, 0]
    half = torch.finfo(HF).eps / 2
    for i, f in enumerate(freqs):
        num, den = f.as_integer_ratio()
        step = (num << (2 * BITS)) // (den * turn)             # turns per position, times 2^BITS
        turns = []
        for p in pos.tolist():
            t = step * p % (1 << BITS)
            turns.append((t - (1 << BITS) if t >> (BITS - 1) else t) / (1 << BITS))
        angle = 2 * math.pi * torch.tensor(turns, dtype=torch.float64)
        for want, at in ((torch.cos(angle), 2 * i if interleaved else i), (torch.sin(angle), 2 * i + 1 if interleaved else rot // 2 + i)):
            want = want * factor
            off = math.pi * 2.0 ** -24 + f * pos.double().abs() * 2.0 ** -52
            tol = (half + 2.0 ** -21) * want.abs() + factor * off * (1 + half) + torch.finfo(HF).tiny * half + factor * 1e-14
            over = (got[:, at] - want).abs() - tol
            assert (over <= 0).all(), f"frequency {f}: {int((over > 0).sum())} over, the worst by {float(over.max()):.3g}"
