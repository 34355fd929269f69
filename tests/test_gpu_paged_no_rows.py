"""sc_paged_append: a sequence that no row joins fits whatever its length says."""
import torch
import pytest

import paged_plain as pp
from paper_2603_14303_b200 import binding

pytestmark = pytest.mark.gpu
DEV = pp.DEV


def test_a_sequence_without_new_rows_is_not_short_of_room():
    """A place of a padded batch that holds no sequence at the moment, its length that of one in a longer table."""
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    k = torch.zeros((4, 1, 4, 8), device=DEV)
    cache = binding.PagedCache(k, k.clone(), torch.arange(4, dtype=torch.int32, device=DEV).view(2, 2))
    new = torch.ones((3, 1, 8), device=DEV)
    status = pp.status_word()
    lens, _ = binding.paged_append(cache, new, new, i32(0, 0, 3), i32(1000, 2), status=status)
    pp.ok(status)
    assert lens.tolist() == [1000, 5] and int(k[:2].count_nonzero()) == 0 and int(k.count_nonzero()) == 24
