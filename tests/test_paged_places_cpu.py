"""Places of a paged session that begin and end, without a device: only their own lengths and counts change."""
import pytest
import torch

from paper_2407_18121_b200.session import PagedCacheSession


def places():
    s = PagedCacheSession.__new__(PagedCacheSession)
    s.N, s.lens, s.seen = 3, torch.tensor([5, 6, -1], dtype=torch.int32), torch.tensor([9, 8, 7], dtype=torch.int32)
    return s


def test_begin_and_end_change_their_own_place():
    s = places()
    s.end(0)
    assert s.lens.tolist() == [-1, 6, -1] and s.seen.tolist() == [9, 8, 7]
    s.begin(0)
    s.begin(2)
    assert s.lens.tolist() == [0, 6, 0] and s.seen.tolist() == [0, 8, 0]


@pytest.mark.parametrize("bad", [-1, 3, 1.0, True, None, torch.tensor(1), [0]])
def test_other_places_are_refused(bad):
    s = places()
    for call in (s.begin, s.end):
        with pytest.raises(ValueError):
            call(bad)
    assert s.lens.tolist() == [5, 6, -1] and s.seen.tolist() == [9, 8, 7]
