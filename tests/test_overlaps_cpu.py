"""Buffers and arrays of one call that share memory: what has no one answer is refused.  No GPU: every call here is refused, or
ends where the library looks for a device."""
import pytest
import torch

from paper_2609_34645_b200 import binding as B
from test_beam_cache_cpu import A, code

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
