"""Append and steps of a paged cache where more rows are protected by their positions than fit: they leave by weight, the
higher candidate first among equals, once all the others have left. Compared bit for bit with the 64-bit form."""
import math

import pytest
import torch

from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from test_paged_gpu import BF, HF, check_append, rand, run_steps

pytestmark = pytest.mark.gpu


def move_positions(m, by, every=1):
    """Adds `by` to the position of every `every`-th row: far behind what has been seen, these rows count as newest."""
    for n, length in enumerate(m.lens.tolist()):
        if length > 0:
            p, s = m.where(n, length)
            m.pos[p[::every], :, s[::every]] += by
    m.dev["pos"].copy_(m.pos)
    return m


def test_eight_new_rows_of_which_seven_count_as_newest():
    m = PagedMirror([0], 1, 64, 16, 16)
    pos = torch.tensor([[[0, 40, 41, 42, 43, 44, 45, 46]]], dtype=torch.int32)
    w = torch.tensor([[[5.0, 1, 2, 3, 4, 5, 6, 7]]])
    check_append(m, 8, 4, recent=2, sinks=1, w=w, pos=pos, fresh=True)
    p, s = m.where(0, 4)
    assert m.pos[p, 0, s].tolist() == [0, 44, 45, 46]


def test_one_new_row_beside_four_that_count_as_newest():
    m = PagedMirror([4], 1, 64, 16, 16)
    p, s = m.where(0, 4)
    for pool in (m.pos, m.dev["pos"]):
        pool[p, 0, s] = torch.tensor([100, 101, 102, 103], dtype=torch.int32, device=pool.device)
    for pool in (m.weight, m.dev["weight"]):
        pool[p, 0, s] = torch.tensor([0.5, 0.1, 0.3, 0.9], dtype=torch.float32, device=pool.device).to(pool.dtype)
    m.weight[p, 0, s] = m.dev["weight"].cpu()[p, 0, s].double()
    for t in (m.seen, m.dev["seen"]):
        t[0] = 4
    check_append(m, 1, 4, recent=2, w=torch.full((1, 1, 1), 0.7))
    assert m.pos[p, 0, s].tolist() == [100, 4, 102, 103]


@pytest.mark.parametrize("every", [1, 2])
@pytest.mark.parametrize("T", [0, 1, 3, 64, 65, 200])
@pytest.mark.parametrize("budget", [300, 120, 7])
def test_more_protected_rows_than_fit(T, every, budget):
    m = move_positions(PagedMirror([300, 299, 0, -1, 40], 2, 64, 16, 304), 5000, every)
    g = torch.Generator().manual_seed(T + budget)
    w = torch.rand(5, 2, T, generator=g) if T else None
    pos = torch.randint(0, 9000, (5, 2, T), generator=g).to(torch.int32) if T > 1 else None
    check_append(m, T, budget, recent=4, sinks=3, w=w, pos=pos)


@pytest.mark.parametrize("T", [1, 90])
@pytest.mark.parametrize("dt,rows", [(BF, "heads"), (HF, "tokens")])
def test_protected_rows_with_equal_and_special_weights(T, dt, rows):
    N, H, L = 2, 3, 400
    m = move_positions(PagedMirror([L, L - 9], H, 64, 24, L, dt, rows), 3000, 2)
    g = torch.Generator().manual_seed(T)
    for n in range(N):
        p, s = m.where(n, int(m.lens[n]))
        fill = torch.randint(0, 3, (len(p), H), generator=g).float()
        fill[::5], fill[1::5], fill[2::7], fill[3::7] = math.inf, -math.inf, math.nan, -0.0
        m.weight[p, :, s] = fill.double()
        m.dev["weight"][p.cuda(), :, s.cuda()] = fill.cuda()
    check_append(m, T, 110, recent=3, sinks=1, w=torch.randint(0, 2, (N, H, T), generator=g).float())


@pytest.mark.parametrize("H,T,budget", [(2, 9000, 300), (1, 20000, 500), (1, 400000, 900), (40, 5000, 64)])
def test_long_prompts_whose_rows_all_count_as_newest(H, T, budget):
    """Lists over one CTA of 1024 threads, over a cluster, over a cluster whose shared memory does not hold them, over many CTAs."""
    m = PagedMirror([0], H, 64, 64, budget)
    g = torch.Generator().manual_seed(T)
    w = torch.exp(torch.randn(1, H, T, generator=g))
    w[:, :, ::3] = 0.25
    check_append(m, T, budget, recent=10, sinks=2, w=w, pos=(torch.arange(T) + T).to(torch.int32).expand(1, H, T).contiguous(), fresh=True)


def test_a_list_beyond_the_clusters_shared_memory_without_protection():
    m = PagedMirror([0], 1, 64, 64, 16000)
    w = torch.exp(torch.randn(1, 1, 400000, generator=torch.Generator().manual_seed(8)))
    check_append(m, 400000, 16000, recent=16, sinks=4, w=w, fresh=True)


@pytest.mark.parametrize("lens,budget,every", [([60, 50, -1, 60], 60, 1), ([60, 57, 0, 60], 20, 2), ([1500, 1490], 1500, 1),
                                               ([2600, 2590], 700, 2)])
@pytest.mark.parametrize("G", [1, 5])
def test_steps_whose_rows_all_count_as_newest(lens, budget, every, G):
    """Half of the weights are negative, so that the new row, which gains at most G, is far from the border of those that leave."""
    m = move_positions(PagedMirror(lens, 3, 64, 16, max(lens) + 4, G=G, ranked=True), 20000, every)
    for n, length in enumerate(lens):
        if length > 0:
            p, s = m.where(n, length)
            m.weight[p, :, s] -= (length // 2) * (G + 1.0)
    m.dev["weight"].copy_(m.weight)
    run_steps(m, G, 4, budget, 6, 2)


def test_a_compacted_cache_with_its_anchors_positions_keeps_the_heaviest():
    """Positions past the rows that were counted, as a compacted cache brings them: all but the lowest count as newest."""
    N, H, keep, budget = 2, 2, 100, 60
    m = PagedMirror([0] * N, H, 64, 16, budget)
    g = torch.Generator().manual_seed(4)
    anchors = torch.stack([torch.randperm(400, generator=g)[:keep].sort().values for _ in range(N * H)]).view(N, H, keep).to(torch.int32)
    check_append(m, keep, budget, recent=8, sinks=1, w=torch.rand(N, H, keep, generator=g), pos=anchors, fresh=True)


def test_protected_rows_with_given_positions_and_a_row_that_cannot_be_read():
    """The rows behind a bad page leave first, protected or not; the others go by weight."""
    m = move_positions(PagedMirror([40], 1, 64, 16, 48), 900)
    m.dev["table"][0, 1] = 1 << 20                                    # rows 16..31
    cache = m.cache(ec)
    old = {k: m.dev[k].clone() for k in ("pos", "weight")}
    K = rand((1, 1, 3, 64), BF, 1).cuda()
    ws = torch.empty(ec.ec_paged_append_workspace(cache, 3, 20), dtype=torch.uint8, device="cuda")
    ec.ec_paged_append(K, K, torch.full((1, 1, 3), 2.0, device="cuda"), None, None, cache, False, 20, 4, 0, ws)
    torch.cuda.synchronize()
    assert ec.ec_device_status(cache._tensors[-1]) == ec.EC_ERR_PAGE and m.dev["lens"].tolist() == [20]
    first = m.table[0, 0].long()
    w = old["weight"][first, 0].cpu()
    got_w, got_p = m.dev["weight"][first, 0].cpu(), m.dev["pos"][first, 0].cpu()
    # 24 readable cached rows and the three new ones, of which 20 stay: the seven lightest leave, some of them of page 0
    third = m.table[0, 2].long()
    every = torch.cat([w, old["weight"][third, 0, :8].cpu(), torch.full((3,), 2.0)])
    keep = set(every.argsort(descending=True, stable=True)[:20].tolist())
    for j in range(16):
        if j in keep:
            assert got_w[j] == w[j] and got_p[j] == old["pos"][first, 0, j].cpu()
        else:
            assert got_p[j] != old["pos"][first, 0, j].cpu()
