"""Books that lie in unusual places."""
import numpy as np
import pytest
import torch

import cache_util as U
from test_gpu_cache import books, ints, seed
from paper_2609_34645_b200 import cache as C

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, columns", [(10, 12), (700, 90)])
def test_two_tables_in_columns_of_one_tensor(rows, columns):
    """A caller that swaps two sets of books keeps both tables in one tensor."""
    rng = seed("columns", rows)
    table, length, refs = books(rng, rows, columns, 4, 3 * rows, 2)
    wide = torch.full((rows, 2 * columns + 1), 99, dtype=torch.int32, device="cuda")
    wide[:, :columns] = ints(table)
    sets = [(wide[:, :columns], ints(length), ints(refs)), (wide[:, columns:2 * columns], ints(length), ints(refs))]
    now = (table, length, refs)
    for step in range(4):
        parent = np.minimum(np.arange(rows) // 2 * 2 + rng.integers(0, 2, rows), rows - 1)
        old, new = sets[step % 2], sets[1 - step % 2]
        got = C.fork([], *old, ints(parent), 4, room=1, out=new)
        want = U.fork(*now, parent, 4, np.ones(rows), rows)
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w)
        now = want[:3]
    got = C.compact([], sets[0][0], sets[0][2], out=(sets[1][0], sets[1][2]))
    want = U.compact(now[0], now[2], None)
    for g, w in ((got[0], want[0]), (got[1], want[1]), (got[2], want[2]), (got[4], want[4])):
        assert np.array_equal(g.cpu().numpy(), w)
    assert (wide[:, 2 * columns] == 99).all()
