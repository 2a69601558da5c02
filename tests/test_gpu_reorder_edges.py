"""States reordered in place where parents cross and lengths end inside a vector: every row gets what its parent held before
the call, to the byte."""
import numpy as np
import pytest
import torch

import cache_util as U
from test_gpu_cache import as_bytes, ints, noise, seed
from paper_2609_34645_b200 import cache as C

pytestmark = pytest.mark.gpu


def check(x, parent, beams, length, dim=1):
    move = (lambda a: a.transpose(0, 2, 1, 3)) if dim == 2 else (lambda a: a)
    old = move(as_bytes(x))
    C.reorder(x, ints(parent), beams=beams, length=ints(length), dim=dim)
    assert np.array_equal(move(as_bytes(x)), U.reorder(old, old, parent, np.asarray(length), beams))


def test_two_rows_swap():
    """66-byte tokens in 132-byte rows: the longer row's third vector of 4 bytes covers the shorter one's last two bytes."""
    x = noise(seed("swap"), (2, 2, 33), torch.bfloat16)
    check(x, [1, 0], 2, [1, 2])
    check(x, [1, 0], 2, [2, 1])


def test_three_rows_heads_first():
    x = noise(seed("heads"), (3, 2, 8, 50), torch.bfloat16)              # tokens of 100 bytes, pieces of 800: vectors of 16
    check(x, [1, 0, 2], 3, [8, 3, 5], dim=2)
    check(x, [2, 0, 1], 3, [1, 7, 3], dim=2)


@pytest.mark.parametrize("beams", [2, 3, 4, 8, 16, 17, 64])
@pytest.mark.parametrize("token", [2, 6, 18, 22, 66, 100, 300])
@pytest.mark.parametrize("unit", [16, 4, 1])
def test_groups_whose_parents_cross(beams, token, unit):
    """Rows whose starts and strides allow vectors of 16, 4 and 1 bytes, tokens that do not; parents are permutations, and any."""
    rng = seed(beams, token, unit)
    tokens, requests = 37, 3
    rows = beams * requests
    stride = -(-tokens * token // unit) * unit + (unit if unit > 1 else 3)
    flat = noise(rng, (rows * stride + 16,), torch.uint8)
    x = torch.as_strided(flat, (rows, tokens, token), (stride, token, 1), 0 if unit == 16 else unit)
    first = np.arange(rows) // beams * beams
    for parent in (np.concatenate([first[r] + rng.permutation(beams) for r in range(0, rows, beams)]), first + rng.integers(0, beams, rows),
                   first + (np.arange(rows) + 1) % beams):
        before = flat.clone()
        check(x, parent, beams, rng.integers(0, tokens + 1, rows))
        gaps = torch.ones(flat.shape[0], dtype=torch.bool, device="cuda")
        torch.as_strided(gaps, x.shape, x.stride(), x.storage_offset()).fill_(False)
        assert torch.equal(flat[gaps], before[gaps])                     # nothing between the rows is written


def test_keys_and_values_of_every_head_side_by_side():
    """Both in place at once, then one to the other's place in the same tensor."""
    rng = seed("side by side")
    whole = noise(rng, (6, 3, 2, 9, 10), torch.bfloat16)                 # rows, heads, keys and values, tokens, width
    states = [whole[:, :, 0], whole[:, :, 1]]
    move = lambda a: a.transpose(0, 2, 1, 3)                             # noqa: E731
    parent, length = [1, 2, 0, 4, 3, 3], np.array([9, 4, 7, 0, 3, 5])
    old = [move(as_bytes(t)) for t in states]
    C.reorder(states, ints(parent), beams=3, length=ints(length), dim=2)
    now = [U.reorder(o, o, parent, length, 3) for o in old]
    for t, w in zip(states, now):
        assert np.array_equal(move(as_bytes(t)), w)
    C.reorder(states[0], ints([5, 5, 0, 1, 2, -1]), length=ints(length), dim=2, out=states[1])
    assert np.array_equal(move(as_bytes(states[0])), now[0])
    assert np.array_equal(move(as_bytes(states[1])), U.reorder(now[0], now[1], [5, 5, 0, 1, 2, -1], length, 0))
