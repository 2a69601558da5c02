"""Buffers and arrays of one call that share memory: what has no one answer is refused.  No GPU: every call here is refused, or
ends where the library looks for a device."""
import pytest
import torch

from paper_2609_34645_b200 import binding as B
from test_beam_cache_cpu import A, NEW, OLD, REST, book, code, pages

FAR = 1 << 34
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused would run on addresses that are none")


def states(bases, rows=4, outer=1, tokens=8, token_bytes=16, row=None, step=0):
    s = B.States(len(bases), rows, outer, tokens, token_bytes, outer * tokens * token_bytes if row is None else row, step)
    for i, b in enumerate(bases):
        s.buffer[i] = b
    return s


def bytes_of(s, base):
    """The bytes of one buffer, one by one."""
    piece = s.tokens * s.token_bytes
    return {base + r * s.row_stride + o * s.outer_stride + k for r in range(s.rows) for o in range(s.outer) for k in range(piece)}


def in_place(s):
    return code(B.states_reorder, s, s, 2, FAR, None)


def test_buffers_that_overlap_in_place():
    for bases in ([A, A], [A, A + 16], [A + 128, A], [A, A + (1 << 20), A + 3 * 128], [A, A + (1 << 20), A]):
        assert in_place(states(bases)) == B.ERR_ALIAS
    assert in_place(states([A, A + 100], row=256)) == B.ERR_ALIAS                         # rows side by side, and not quite
    assert in_place(states([A, A + 64], outer=2, tokens=8, row=512, step=256)) == B.ERR_ALIAS
    assert in_place(states([A, A + 128], outer=2, row=384, step=256)) == B.ERR_ALIAS        # meets the next row's


def test_written_buffers_that_overlap_out_of_place():
    src = states([A, A + (1 << 20)])
    for bases in ([FAR, FAR], [FAR, FAR + 8], [FAR + 384, FAR]):
        assert code(B.states_reorder, src, states(bases), 0, FAR - 4096, None) == B.ERR_ALIAS


@no_gpu
def test_what_lies_side_by_side_is_taken():
    for bases, kw in (([A, A + 512], {}), ([A, A + 128, A + 256], dict(row=384)), ([A + 256, A, A + 128], dict(row=384)),
                      ([A, A + 128], dict(outer=2, row=512, step=256)),                    # keys and values of every head
                      ([A, A + 128, A + 1024, A + 1152], dict(outer=4, row=2048, step=256)),
                      ([A, A + 4096, A + 128, A + 4096 + 128], dict(row=256)), ([A, A + 64], dict(outer=2, tokens=4, row=128, step=512))):
        assert in_place(states(bases, **kw)) == B.ERR_CUDA
    assert code(B.states_reorder, states([A, A]), states([FAR, FAR]), 0, FAR + 4096, None) == B.ERR_CUDA         # one buffer, named twice


@no_gpu
def test_overlaps_are_told_byte_by_byte():
    import random
    rng = random.Random(5)
    told = {B.ERR_ALIAS: 0, B.ERR_CUDA: 0}
    for _ in range(4000):
        rows, outer, tokens, token_bytes = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 3), rng.choice([1, 2, 5])
        rows *= 2
        piece = tokens * token_bytes
        if rng.random() < 0.5:
            step = rng.randint(piece, 3 * piece)
            row = rng.randint((outer - 1) * step + piece, 3 * outer * step)
        else:
            row = rng.randint(piece, 3 * piece)
            step = rng.randint((rows - 1) * row + piece, 3 * rows * row)
        hull = (rows - 1) * row + (outer - 1) * step + piece
        s = states([A + rng.randint(0, rng.choice([piece * 4, hull * 2, hull * 6])) for _ in range(rng.randint(2, 4))], rows, outer, tokens, token_bytes,
                   row, step)
        held, n = set(), 0
        for i in range(s.buffers):
            held |= bytes_of(s, s.buffer[i])
            n += rows * outer * piece
        want = B.ERR_CUDA if len(held) == n else B.ERR_ALIAS
        assert in_place(s) == want, (list(s.buffer[:s.buffers]), rows, outer, piece, row, step)
        told[want] += 1
    assert min(told.values()) > 500


# ---- arrays within buffers, pools that overlap -------------------------------------------------------------------

def test_arrays_within_the_states_that_are_written():
    s = states([A, A + (1 << 20)], row=256)
    for at in (A, A + 4, A + 124, A + 3 * 256 + 120, A + (1 << 20) + 512, A - 12):
        assert code(B.states_reorder, s, s, 2, at, None) == code(B.states_reorder, s, s, 2, FAR, at) == B.ERR_ALIAS
    src = states([FAR << 1, (FAR << 1) + (1 << 20)], row=256)
    assert code(B.states_reorder, src, s, 0, A + 8, None) == B.ERR_ALIAS


def test_arrays_within_the_pools():
    def fork(old=None, new=None, parent=REST, room_of=None, copies=REST + 4096, status=REST + 8192, pool=None):
        return code(B.cache_fork, pool or pages(), old or book(OLD), new or book(NEW), parent, 16, 0, room_of, copies, status)

    def compact(old=None, new=None, where=REST, moves=REST + 4096, status=REST + 8192, pool=None):
        return code(B.cache_compact, pool or pages(), old or book(OLD), new or book(NEW), -1, where, moves, status)
    for at in (A, A + 636, A + (1 << 16) + 64):                                            # pages are 640 bytes of each pool
        for call in (fork, compact):
            assert call(old=book(OLD, table=at)) == call(old=book(OLD, refs=at)) == call(new=book(NEW, table=at)) == B.ERR_ALIAS
            assert call(new=book(NEW, refs=at)) == call(status=at) == B.ERR_ALIAS
        assert fork(old=book(OLD, length=at)) == fork(new=book(NEW, length=at)) == fork(parent=at) == fork(room_of=at) == fork(copies=at) == B.ERR_ALIAS
        assert compact(where=at) == compact(moves=at - at % 8) == B.ERR_ALIAS
        assert code(B.cache_copy, pages(base=OLD), pages(), 3, at, REST) == code(B.cache_copy, pages(), pages(), 3, REST, at) == B.ERR_ALIAS


def test_pools_that_overlap():
    shifted = pages()
    shifted.pool[1] = shifted.pool[0] + 64                                                 # page p of one is page p + 1 of the other
    assert code(B.cache_fork, shifted, book(OLD), book(NEW), REST, 16, 0, None, REST + 4096, REST + 8192) == B.ERR_ALIAS
    assert code(B.cache_compact, shifted, book(OLD), book(NEW), -1, REST, REST + 4096, REST + 8192) == B.ERR_ALIAS
    assert code(B.cache_copy, shifted, shifted, 3, REST, REST + 4096) == code(B.cache_copy, pages(base=OLD), shifted, 3, REST, REST + 4096) == B.ERR_ALIAS
    twice = pages()
    twice.pool[1] = twice.pool[0]
    assert code(B.cache_copy, pages(base=OLD), twice, 3, REST, REST + 4096) == B.ERR_ALIAS


@no_gpu
def test_arrays_and_pools_that_do_not_meet():
    twice = pages()
    twice.pool[1] = twice.pool[0]                                                          # one pool, named twice
    assert code(B.cache_copy, twice, twice, 3, REST, REST + 4096) == B.ERR_CUDA
    wide = pages(stride=128)
    wide.pool[1] = wide.pool[0] + 64                                                       # keys and values of a page side by side
    assert code(B.cache_fork, wide, book(OLD), book(NEW), REST, 16, 0, None, REST + 4096, REST + 8192) == B.ERR_CUDA
    gap = pages(stride=128)
    assert code(B.cache_copy, gap, gap, 3, A + 64, A + 128 + 64) == B.ERR_CUDA             # arrays between two pages
    assert code(B.cache_copy, gap, gap, 17, A + 64, REST) == B.ERR_ALIAS                   # 17 numbers reach the next
    s = states([A], row=256)
    assert code(B.states_reorder, s, s, 2, A + 128, A + 256 + 128) == B.ERR_CUDA


# ---- tables that are columns of one tensor -----------------------------------------------------------------------

def fork_of(old, new, parent=REST, copies=REST + 4096):
    return code(B.cache_fork, pages(), old, new, parent, 16, 0, None, copies, REST + 8192)


def compact_of(old, new):
    return code(B.cache_compact, pages(), old, new, -1, REST, REST + 4096, REST + 8192)


def test_tables_that_share_columns():
    for at, stride in ((OLD + 12, 8), (OLD + 32 * 2 + 12, 8), (OLD + 20, 8), (OLD + 16, 9), (OLD + 8, 4), (OLD + 64, 8)):
        new = book(NEW, table=at, stride=stride)
        assert fork_of(book(OLD, stride=8), new) == compact_of(book(OLD, stride=8), new) == B.ERR_ALIAS
    # an array within a row of either table
    assert fork_of(book(OLD, stride=8), book(NEW, stride=8), copies=OLD + 32) == fork_of(book(OLD, stride=8), book(NEW, stride=8), parent=NEW + 12) == B.ERR_ALIAS


@no_gpu
def test_tables_side_by_side():
    for at in (OLD + 16, OLD - 16, OLD + 32 + 16):
        new = book(NEW, table=at, stride=8)
        assert fork_of(book(OLD, stride=8), new) == compact_of(book(OLD, stride=8), new) == B.ERR_CUDA
    assert fork_of(book(OLD, rows=1), book(NEW, rows=1, table=OLD + 16)) == B.ERR_CUDA
    assert fork_of(book(OLD, stride=8), book(NEW, stride=8), parent=NEW + 16) == B.ERR_CUDA


# ---- out of place, between buffers of one tensor -------------------------------------------------------------------

@no_gpu
def test_from_one_buffer_to_another_between_its_pieces():
    def move(src, dst):
        return code(B.states_reorder, src, dst, 0, FAR, None)
    keys, values = states([A], outer=2, row=512, step=256), states([A + 128], outer=2, row=512, step=256)      # of every head
    assert move(keys, values) == move(values, keys) == B.ERR_CUDA
    assert move(keys, states([A + 128], rows=2, outer=2, row=512, step=256)) == move(states([A], rows=1, outer=2, step=256), values) == B.ERR_CUDA
    assert move(keys, states([A + 127], outer=2, row=512, step=256)) == move(keys, states([A + 129], outer=2, row=512, step=256)) == B.ERR_ALIAS
    assert move(keys, states([A + 512], outer=2, row=512, step=256)) == B.ERR_ALIAS                              # a row further on
    import random
    rng = random.Random(9)
    told = {B.ERR_ALIAS: 0, B.ERR_CUDA: 0}
    for _ in range(4000):
        rows, more, outer, piece = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 4), rng.choice([1, 2, 5])
        if rng.random() < 0.5:
            step = rng.randint(piece, 3 * piece)
            row = rng.randint((outer - 1) * step + piece, 3 * outer * step)
        else:
            row = rng.randint(piece, 3 * piece)
            step = rng.randint((max(rows, more) - 1) * row + piece, 3 * max(rows, more) * row)
        hull = (rows - 1) * row + (outer - 1) * step + piece
        far = rng.choice([piece * 4, hull * 2])
        src = states([A + rng.randint(0, far) for _ in range(2)], rows, outer, 1, piece, row, step)
        dst = states([A + rng.randint(0, far), A + (1 << 20)], more, outer, 1, piece, row, step)
        if src.buffer[0] == dst.buffer[0]:
            continue
        held = bytes_of(src, src.buffer[0]) | bytes_of(src, src.buffer[1])
        want = B.ERR_ALIAS if held & bytes_of(dst, dst.buffer[0]) else B.ERR_CUDA
        assert move(src, dst) == want, (src.buffer[0], src.buffer[1], dst.buffer[0], rows, more, outer, piece, row, step)
        told[want] += 1
    assert min(told.values()) > 500
