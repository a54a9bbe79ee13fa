"""Calls on a paged cache that its documentation allows and the other tests do not make."""
import pytest
import torch

from paged_reference import PagedMirror
from paper_2407_18121_b200 import binding as ec
from test_paged_gpu import BF, HF, check_append, rand, run_steps, state_of
from test_paged_precision_gpu import check
from test_paged_protected_gpu import move_positions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [2, 40, 64])
@pytest.mark.parametrize("budget,every", [(16500, 0), (16400, 0), (16500, 1), (9000, 2)])
def test_few_rows_onto_lists_that_a_cluster_shares(T, budget, every):
    """Selected by eight CTAs, which move the rows themselves."""
    m = PagedMirror([16500, 16488], 2, 64, 64, 16512)
    if every:
        move_positions(m, 60000, every)
    w = torch.rand(2, 2, T, generator=torch.Generator().manual_seed(T))
    check_append(m, T, budget, recent=min(T, 20), sinks=3, w=w)


@pytest.mark.parametrize("page,budget", [(64, 20000), (4, 3000)])
def test_steps_far_below_the_budget(page, budget):
    """A table and a budget that reach much further than the sequences: most of the rows launch has nothing to do."""
    m = PagedMirror([10, 0, 700, -1], 2, 64, page, budget, G=2, ranked=True)
    run_steps(m, 2, 4, budget, 4, 1)


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("scale", [1e-12, 1e-30, 1e-38])
def test_scales_under_which_all_rows_are_alike(dt, scale):
    m = PagedMirror([100, 1, 0, 300], 2, 64, 16, 304, dt)
    q, k, v = (rand((4, h, 64), dt, 50 + h) for h in (6, 2, 2))
    check(m, q, k, v, scale)


@pytest.mark.parametrize("T", [0, 1])
def test_a_fresh_start_with_one_row_or_none(T):
    m = PagedMirror([40, 0, -1, 7], 2, 64, 16, 48)
    w = torch.rand(4, 2, T, generator=torch.Generator().manual_seed(T)) if T else None
    check_append(m, T, 32, recent=1, w=w, fresh=True, counts=torch.tensor([T, 1, T, 0], dtype=torch.int32))


def test_keys_and_values_side_by_side_in_one_tensor():
    m = PagedMirror([90, 33], 3, 64, 16, 96, G=2, ranked=True)
    n_pages = m.K.shape[0]
    both = torch.empty(n_pages, 16, 3, 2, 64, dtype=BF, device="cuda")        # a page holds slot by slot every head's key and value
    for i, name in enumerate(("K", "V")):
        view = both[:, :, :, i].transpose(1, 2)
        view.copy_(m.dev[name])
        m.dev[name] = view
    run_steps(m, 2, 4, 96, 6, 1)


def test_a_step_repeated_from_one_state_gives_the_same_bits():
    outs = []
    for _ in range(3):
        m = PagedMirror([900, 31, 640], 8, 128, 16, 900, HF, G=5, ranked=True)
        cache = m.cache(ec)
        ws = torch.empty(ec.ec_paged_step_workspace(cache, 40, 900), dtype=torch.uint8, device="cuda")
        q, k, v = (rand((3, h, 128), HF, h).cuda() for h in (40, 8, 8))
        out, lse = torch.empty_like(q), torch.empty(3, 40, device="cuda")
        for _ in range(5):
            ec.ec_paged_decode_step(q, k, v, cache, 0.0884, 0.9, 900, 8, 2, out, lse, ws)
        torch.cuda.synchronize()
        assert ec.ec_device_status(state_of(cache)) == ec.EC_OK
        outs.append([t.clone().nan_to_num(7.0) for t in (out, lse, m.dev["weight"], m.dev["K"])] + [m.dev["pos"].clone()])
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a, b)
