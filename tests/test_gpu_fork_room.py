"""Forks that hand out thousands of fresh pages, as when room is made for prompts: more than a block ranks at a time, over free
pages that lie scattered, so that a window of them ends inside a group."""
import numpy as np
import pytest
import torch

from test_gpu_cache import check_fork, ints, noise, seed
from paper_2609_34645_b200 import cache as C

pytestmark = pytest.mark.gpu


def scattered(rng, rows, columns, page_size, pages, live, tokens):
    """Sequences of `tokens` tokens on pages in no order; of the other pages a share `live` is held by somebody else."""
    held = -(-tokens // page_size)
    name = rng.permutation(pages)
    table = np.full((rows, columns), -1)
    table[:, :held] = name[:rows * held].reshape(rows, held)
    refs = (rng.random(pages) < live).astype(np.int64)
    refs[table[table >= 0]] = 1
    return table, np.full(rows, tokens), refs


# rows, columns, page_size, pages, share of the pages that others hold, tokens of a row, room, fresh pages at least
ROOMS = [(2, 2001, 16, 30000, 0.5, 5, 31990, 3990),              # small books: one block does it all
         (2, 2000, 16, 30000, 0.01, 0, 32000, 4000),
         (512, 40, 8, 30000, 0.5, 13, 40, 2500),                 # one block ranks
         (1024, 40, 16, 6000, 0.0, 32, 40, 3000),
         (300, 90, 16, 32768, 0.1, 1, 1100, 20000),
         (64, 800, 4, 120000, 0.5, 9, 3180, 50000),              # a cluster does
         (40, 1300, 16, 70000, 0.02, 20, 20700, 51000)]


@pytest.mark.parametrize("shape", ROOMS)
def test_room_for_prompts(shape):
    rows, columns, page_size, pages, live, tokens, room, least = shape
    rng = seed(shape)
    table, length, refs = scattered(rng, rows, columns, page_size, pages, live, tokens)
    for parent in (np.arange(rows), np.arange(rows) // 2 * 2):
        status = check_fork(rng, table, length, refs, parent, page_size, room)[4]
        assert status[1] == 0
        # nothing that is handed out is anybody else's
        new, _, counts, _, _ = C.fork([], ints(table), ints(length), ints(refs), ints(parent), page_size, room=room)
        new, counts = new.cpu().numpy(), counts.cpu().numpy()
        fresh = new[(new >= 0) & ~np.isin(new, table)]
        if parent[1] == 1:                                               # nothing was released that could be handed out again
            assert len(fresh) >= least
        assert len(set(fresh.tolist())) == len(fresh) and (counts[fresh] == 1).all() and (refs[fresh] == 0).all()


@pytest.mark.parametrize("pages", [9000, 12000, 60000])                 # 9000 are not enough
def test_room_differs_from_row_to_row(pages):
    """Rows that have pages behind a gap, rows that need none, copies of begun pages among what is handed out."""
    rng = seed("rows", pages)
    table, length, refs = scattered(rng, 200, 60, 8, pages, 0.3, 21)
    length = rng.integers(0, 25, 200)
    gaps = rng.random(200) < 0.3
    table[gaps, 30] = np.flatnonzero(refs == 0)[:int(gaps.sum())]
    refs[table[gaps, 30]] = 1
    parent = rng.integers(0, 200, 230)
    pool = noise(rng, (len(refs), 24), torch.bfloat16)
    room = np.where(rng.random(230) < 0.2, 0, rng.integers(100, 400, 230))
    want = check_fork(rng, table, length, refs, parent, 8, 0, [pool], room)
    assert (want[4][1] > 0) == (pages == 9000) and (want[4][2] > 20) == (pages > 9000)
