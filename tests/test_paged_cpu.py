"""Host-side checks of the paged cache's entry points: refusals, workspace sizes, the look over a page table, and the
plain forms the GPU tests compare with."""
import ctypes as C

import pytest
import torch

from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from paper_2407_18121_b200 import build as ecbuild

P = 0x10000          # aligned, never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def L():
    ecbuild.build()
    return ec.lib()


def paged(**kw):
    c = ec.ec_paged()
    v = dict(Kp=P, Vp=P, weight=P, pos=P, table=P, lens=P, seen=P, state=P, N=2, H=3, D=64, page_size=16, n_pages=10,
             max_pages=4, dtype=0, page_stride=3 * 16 * 64, head_stride=16 * 64, row_stride=64)
    v.update(kw)
    for k, x in v.items():
        setattr(c, k, x)
    return c


BAD = [(dict(Kp=None), 1), (dict(weight=None), 1), (dict(lens=None), 1), (dict(state=None), 1), (dict(N=0), 2), (dict(H=0), 2),
       (dict(D=96), 2), (dict(page_size=0), 2), (dict(n_pages=0), 2), (dict(max_pages=0), 2), (dict(N=1 << 20, H=16), 2),
       (dict(max_pages=1 << 20, page_size=1 << 12), 2), (dict(n_pages=1 << 20, H=64, page_size=64), 2), (dict(dtype=2), 4),
       (dict(row_stride=56), 4), (dict(row_stride=68), 4), (dict(page_stride=-64), 4), (dict(head_stride=0), 4),
       (dict(page_stride=1 << 34), 2), (dict(Kp=P + 8), 3), (dict(pos=P + 2), 3), (dict(state=P + 16), 3)]


@pytest.mark.parametrize("bad,status", BAD)
def test_a_bad_description_is_refused_everywhere(L, bad, status):
    c = paged(**bad)
    big = 1 << 40
    fields = [getattr(c, n) for n, _ in ec.ec_paged._fields_]
    d = ec.ec_paged()
    assert L.ec_paged_init(C.byref(d), *fields[:8], *fields[8:15], *fields[15:], None) == status
    assert L.ec_paged_attention(P, P, P, C.byref(c), 6, 1.0, 0, 1.0, P, None, None, P, big, None) == status
    assert L.ec_paged_append(P, P, None, None, None, C.byref(c), 1, 0, 8, 1, 0, P, big, None) == status
    assert L.ec_paged_decode_step(P, P, P, C.byref(c), 6, 1.0, 1.0, 8, 1, 0, P, None, P, big, None) == status
    assert L.ec_paged_attention_workspace(C.byref(c), 6, 1) == 0
    assert L.ec_paged_append_workspace(C.byref(c), 1, 8) == 0
    assert L.ec_paged_step_workspace(C.byref(c), 6, 8) == 0


def test_attention_refusals(L):
    c, ws = paged(), 1 << 40
    r = C.byref(c)
    f = L.ec_paged_attention
    assert f(None, P, P, r, 6, 1.0, 0, 1.0, P, None, None, P, ws, None) == 1
    assert f(P, P, None, r, 6, 1.0, 0, 1.0, P, None, None, P, ws, None) == 1          # k_new without v_new
    assert f(P, P, P, r, 6, 1.0, 0, 1.0, None, None, None, P, ws, None) == 1
    assert f(P, P, P, r, 6, 1.0, 1, 1.0, P, None, None, P, ws, None) == 1             # w_new missing
    assert f(P, P, P, None, 6, 1.0, 0, 1.0, P, None, None, P, ws, None) == 1
    assert f(P, P, P, r, 7, 1.0, 0, 1.0, P, None, None, P, ws, None) == 2             # Hq not a multiple of H
    assert f(P, P, P, r, 0, 1.0, 0, 1.0, P, None, None, P, ws, None) == 2
    assert f(P, P, P, r, 3 * 129, 1.0, 0, 1.0, P, None, None, P, ws, None) == 2       # group too wide
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert f(P, P, P, r, 6, scale, 0, 1.0, P, None, None, P, ws, None) == 4
    for decay in (0.0, 1.5, float("nan")):
        assert f(P, P, P, r, 6, 1.0, 1, decay, P, None, P, P, ws, None) == 4
    assert f(P + 8, P, P, r, 6, 1.0, 0, 1.0, P, None, None, P, ws, None) == 3
    assert f(P, P, P, r, 6, 1.0, 0, 1.0, P, P + 2, None, P, ws, None) == 3
    assert f(P, P, P, r, 6, 1.0, 0, 1.0, P, None, None, None, 0, None) == 5
    assert f(P, P, P, r, 6, 1.0, 0, 1.0, P, None, None, P, 64, None) == 5
    assert f(P, P, P, r, 6, 1.0, 0, 1.0, P, None, None, P + 64, ws, None) == 3
    assert L.ec_paged_attention_workspace(r, 7, 0) == 0
    # gathered weights need a score per row and query head
    assert L.ec_paged_attention_workspace(r, 6, 1) >= L.ec_paged_attention_workspace(r, 6, 0) + 10 * 16 * 6 * 4


def test_a_scale_whose_log2_form_overflows_is_refused(L):
    c = paged()
    for accumulate, w_new in ((0, None), (1, P)):
        assert L.ec_paged_attention(P, P, P, C.byref(c), 6, 3e38, accumulate, 1.0, P, None, w_new, P, 1 << 40, None) == 4


def test_append_and_step_refusals(L):
    c, ws = paged(), 1 << 40
    r = C.byref(c)
    f = L.ec_paged_append
    assert f(None, P, None, None, None, r, 1, 0, 8, 1, 0, P, ws, None) == 1
    assert f(P, None, None, None, None, r, 1, 0, 8, 1, 0, P, ws, None) == 1
    assert f(P, P, None, None, None, r, -1, 0, 8, 1, 0, P, ws, None) == 4
    assert f(P, P, None, None, None, r, 1, 0, 0, 0, 0, P, ws, None) == 4              # budget
    assert f(P, P, None, None, None, r, 1, 0, 65, 0, 0, P, ws, None) == 4             # beyond the table
    assert f(P, P, None, None, None, r, 1, 0, 8, 5, 4, P, ws, None) == 4              # protects more than the budget
    assert f(P, P, None, None, None, r, 1, 0, 8, -1, 0, P, ws, None) == 4
    assert f(P, P, None, None, None, r, 1 << 30, 0, 8, 1, 0, P, ws, None) == 2
    assert f(P + 4, P, None, None, None, r, 1, 0, 8, 1, 0, P, ws, None) == 3
    assert f(P, P, P + 1, None, None, r, 1, 0, 8, 1, 0, P, ws, None) == 3
    assert f(P, P, None, None, None, r, 1, 0, 8, 1, 0, P, 16, None) == 5
    g = L.ec_paged_decode_step
    assert g(P, None, None, r, 6, 1.0, 1.0, 8, 1, 0, P, None, P, ws, None) == 1
    assert g(P, P, P, r, 6, 1.0, 0.0, 8, 1, 0, P, None, P, ws, None) == 4
    assert g(P, P, P, r, 6, 1.0, 1.0, 8, 9, 0, P, None, P, ws, None) == 4
    assert g(P, P, P, r, 6, 1.0, 1.0, 8, 1, 0, P, None, P, L.ec_paged_step_workspace(r, 6, 8) - 1, None) == 5
    assert L.ec_paged_state_bytes(0) == 0 and L.ec_paged_state_bytes(100) >= 256 + 400
    assert ec.status_string(ec.EC_ERR_PAGE) not in ("unknown status", ec.status_string(ec.EC_OK))


def test_check_finds_bad_tables(L):
    c = paged()

    def check(table, lens, rows=0):
        try:
            ec.ec_paged_check(c, torch.tensor(table, dtype=torch.int32), torch.tensor(lens, dtype=torch.int32), rows)
        except ec.EcError as e:
            return e.status
        return 0
    good = [[0, 1, 2, 3], [4, 5, 6, 7]]
    assert check(good, [64, 64]) == 0
    assert check(good, [65, 0]) == 9                                       # a length beyond the table
    assert check([[0, 1, 2, 10], [4, 5, 6, 7]], [64, 1]) == 9              # outside the pool
    assert check([[0, 1, 2, -1], [4, 5, 6, 7]], [48, 1]) == 0              # not reached
    assert check([[0, 1, 2, -1], [4, 5, 6, 7]], [48, 1], rows=49) == 9     # reached when it grows
    assert check([[0, 1, 2, 3], [4, 1, 6, 7]], [64, 17]) == 9              # one page, two places
    assert check([[0, 1, 2, 3], [4, 1, 6, 7]], [64, 16]) == 0
    assert check([[0, 1, 2, 3], [99, 99, 99, 99]], [64, -1], rows=64) == 0  # an empty place
    assert check(good, [1, 1], rows=65) == 4


def test_plain_append_keeps_what_the_definition_keeps():
    """The mirror's own rule on a case worked by hand: 4 rows, budget 4, one new row."""
    m = PagedMirror([4], 1, 64, 2, 4, device=None)
    p, s = m.where(0, 4)
    m.weight[p, 0, s] = torch.tensor([0.5, 0.1, 0.1, 0.9], dtype=torch.float64)
    m.pos[p, 0, s] = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    m.seen[0] = 4
    row = torch.ones(1, 1, 1, 64, dtype=torch.bfloat16)
    m.append(row, row, torch.full((1, 1, 1), 0.05), None, None, 1, False, 4, 1, 0)
    # rows 1 and 2 are equal: the higher one leaves; the new row (protected) takes its place
    assert m.pos[p, 0, s].tolist() == [0, 1, 4, 3] and int(m.lens[0]) == 4 and int(m.seen[0]) == 5
    assert m.K[p[2], 0, s[2]].eq(1).all()
    m.append(row, row, torch.full((1, 1, 1), 0.07), None, None, 1, False, 3, 0, 0)
    # now 0.05 and 0.07 leave; the row behind the new length moves into the hole
    assert m.pos[p[:3], 0, s[:3]].tolist() == [0, 1, 3] and int(m.lens[0]) == 3


def test_plain_attention_matches_a_library_softmax():
    m = PagedMirror([9, 0], 2, 64, 4, 12, device=None)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(2, h, 64, generator=g).bfloat16() for h in (4, 2, 2))
    (out, lse, w_new), _, _ = m.attention(q, k, v, 0.125, True)
    p, s = m.where(0, 9)
    K = torch.cat([m.K[p, :, s], k[0][None]]).double().repeat_interleave(2, 1).transpose(0, 1)
    V = torch.cat([m.V[p, :, s], v[0][None]]).double().repeat_interleave(2, 1).transpose(0, 1)
    x = (K @ q[0].double()[..., None])[..., 0] * 0.125
    want = torch.softmax(x, -1)
    assert torch.allclose(out[0], (want[:, None] @ V)[:, 0]) and torch.allclose(lse[0], torch.logsumexp(x, -1))
    assert torch.allclose(w_new[0], want[:, -1].view(2, 2).sum(1))
    assert torch.equal(out[1].view(2, 2, 64)[:, 0], v[1].double()) and torch.equal(w_new[1], torch.full((2,), 2.0, dtype=torch.float64))
