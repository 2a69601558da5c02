"""States and paged caches against their definitions (tests/cache_util.py): everything is moved or counted, so that every
result is equal."""
import zlib

import numpy as np
import pytest
import torch

import cache_util as U
from paper_2609_34645_b200 import binding as B
from paper_2609_34645_b200 import cache as C

pytestmark = pytest.mark.gpu


def seed(*key):
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def ints(a):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda", torch.int32)


def noise(rng, shape, dtype):
    """A tensor of random bytes."""
    size = torch.empty(0, dtype=dtype).element_size()
    raw = rng.integers(0, 256, (*shape[:-1], shape[-1] * size), dtype=np.uint8)
    return torch.as_tensor(raw).cuda().view(dtype)


def as_bytes(t):
    t = t.contiguous()
    return t.view(torch.uint8).cpu().numpy().reshape(*t.shape[:-1], -1) if t.dim() > 1 else t.view(torch.uint8).cpu().numpy()


# ---- reorder ---------------------------------------------------------------------------------------------------

# requests, beams, tokens, heads, width
STATES = [(1, 1, 1, 1, 1), (1, 4, 300, 2, 64), (3, 5, 37, 3, 50), (2, 8, 129, 1, 7), (1, 64, 33, 2, 16), (2, 33, 5, 1, 3), (4, 12, 70, 1, 128),
          (2, 16, 1025, 1, 9), (7, 3, 2, 5, 33)]


@pytest.mark.parametrize("shape", STATES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.uint8])
@pytest.mark.parametrize("layout", ["tokens", "heads", "slices", "odd"])
def test_reorder_in_place(shape, dtype, layout):
    """Parents that cross, stay, name another group or no row; lengths outside the tokens; views of a wider tensor."""
    requests, beams, tokens, heads, width = shape
    rng = seed(shape, dtype, layout)
    rows = requests * beams
    local = rng.integers(0, beams, rows)
    parent = local + np.arange(rows) // beams * beams
    odd = rng.random(rows)
    parent[odd < 0.1] = -1
    parent[(odd >= 0.1) & (odd < 0.2)] = rng.integers(0, rows + 3)
    for length in (None, rng.integers(-2, tokens + 3, rows)):
        if layout == "heads":
            whole = noise(rng, (3, rows, heads, tokens, width), dtype)
            states, dim = list(whole.unbind(0)), 2
            plain = [as_bytes(t).transpose(0, 2, 1, 3) for t in states]
        elif layout == "tokens":
            whole = noise(rng, (3, rows, tokens, heads, width), dtype)
            states, dim = list(whole.unbind(0)), 1
            plain = [as_bytes(t) for t in states]
        elif layout == "slices":                     # keys and values side by side in a row
            whole = noise(rng, (rows, 2, tokens, heads, width), dtype)
            states, dim = [whole[:, 0], whole[:, 1]], 1
            plain = [as_bytes(t) for t in states]
        else:                                        # off by an element, rows of an odd stride
            flat = noise(rng, (rows * (tokens * heads * width + 3) + 5,), dtype)
            whole = flat
            states = [torch.as_strided(flat, (rows, tokens, heads, width), (tokens * heads * width + 3, heads * width, width, 1), 1)]
            dim = 1
            plain = [as_bytes(t) for t in states]
        before = whole.clone()
        assert C.reorder(states, ints(parent), beams=beams, length=None if length is None else ints(length), dim=dim) is states
        for t, old in zip(states, plain):
            want = U.reorder(old, old, parent, length, beams)
            got = as_bytes(t).transpose(0, 2, 1, 3) if layout == "heads" else as_bytes(t)
            assert np.array_equal(got, want)
        if layout == "odd":                          # nothing between the rows is written
            for t in (whole, before):
                torch.as_strided(t, states[0].shape, states[0].stride(), 1).zero_()
            assert torch.equal(whole.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("rows", [1, 4, 37, 130])
@pytest.mark.parametrize("from_rows", [1, 3, 50])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_reorder_to_other_buffers(rows, from_rows, dtype):
    rng = seed(rows, from_rows, dtype)
    tokens, heads, width = 61, 2, 24
    whole = noise(rng, (5, from_rows, heads, tokens, width), dtype)
    out = noise(rng, (5, rows, heads, tokens, width), dtype)
    parent = rng.integers(-1, from_rows + 1, rows)
    length = rng.integers(0, tokens + 1, from_rows)
    old, new = as_bytes(whole).transpose(0, 1, 3, 2, 4), as_bytes(out).transpose(0, 1, 3, 2, 4)
    states, to = list(whole.unbind(0)), list(out.unbind(0))
    assert C.reorder(states, ints(parent), length=ints(length), dim=2, out=to) is to
    got = as_bytes(out).transpose(0, 1, 3, 2, 4)
    for b in range(5):
        assert np.array_equal(got[b], U.reorder(old[b], new[b], parent, length, 0))
    assert np.array_equal(as_bytes(whole).transpose(0, 1, 3, 2, 4), old)


def test_reorder_one_tensor_without_tokens():
    rng = seed("plain")
    x = noise(rng, (6, 1000), torch.float32)
    y, parent = x.clone(), ints([1, 0, 0, 5, 4, 3])
    C.reorder(x, parent, beams=3)
    assert np.array_equal(as_bytes(x), as_bytes(y[parent.long()]))        # random bytes: some are NaN
    score, order = torch.arange(6, device="cuda", dtype=torch.float32), ints([2, 2, 1, 4, 3, 3])
    C.reorder(score, order, beams=3)
    assert score.tolist() == [2, 2, 1, 4, 3, 3]
    C.reorder(x[:0], ints([]), beams=3)
    C.reorder(x[:, :0], parent, beams=3)
    out = torch.zeros(6, 1000, device="cuda")
    C.reorder(x, parent, out=out)
    assert np.array_equal(as_bytes(out), as_bytes(x[parent.long()]))


def test_reorder_past_32_bits():
    """Rows that lie more than 4 GiB apart."""
    rows, width = 3, (1 << 32) + 48
    if torch.cuda.mem_get_info()[0] < 3 * width + (8 << 30):
        pytest.skip("needs 20 GiB")
    x = torch.zeros(rows, width, dtype=torch.uint8, device="cuda")
    for r in range(rows):
        x[r, -40:] = r + 1
        x[r, :40] = 10 * (r + 1)
    C.reorder(x, ints([0, 2, 0]), beams=3)
    assert x[:, -1].tolist() == [1, 3, 1] and x[:, 0].tolist() == [10, 30, 10] and int(x[1, width // 2]) == 0


# ---- fork ------------------------------------------------------------------------------------------------------

def books(rng, rows, columns, page_size, spare, share):
    """A page table of sequences that begin alike in groups of `share`, lengths of any kind among them, pages in no order."""
    length = rng.integers(0, columns * page_size + 1, rows)
    length[rng.random(rows) < 0.2] = 0
    length[rng.random(rows) < 0.2] //= max(page_size, 1)
    at, table = 0, np.full((rows, columns), -1)
    for r in range(rows):
        held = -(-int(length[r]) // page_size)
        first = r // share * share
        common = 0 if r == first else min(int(length[r]), int(length[first])) // page_size // 2
        table[r, :common] = table[first, :common]
        more = min(columns, held + (rng.integers(0, 3) if rng.random() < 0.3 else 0))       # room that was made before
        table[r, common:more] = np.arange(at, at + more - common)
        at += more - common
    pages = at + spare
    name = rng.permutation(max(pages, 1))
    table = np.where(table >= 0, name[np.maximum(table, 0)], -1)
    refs = np.bincount(table[table >= 0], minlength=max(pages, 1))
    return table, length, refs


def check_fork(rng, table, length, refs, parent, page_size, room, pools=None, room_of=None):
    rows = len(parent)
    held = [] if pools is None else pools
    old = [as_bytes(p) for p in held]
    got = C.fork(held, ints(table), ints(length), ints(refs), ints(parent), page_size,
                 room=room if room_of is None else ints(room_of))
    want = U.fork(table, length, refs, parent, page_size, np.full(rows, room) if room_of is None else room_of, rows)
    for g, w, what in zip(got, want, ("table", "length", "refs", "copies", "status")):
        assert np.array_equal(g.cpu().numpy(), w), what
    for p, o in zip(held, old):
        for a, b in want[3]:
            if b >= 0:
                o[b] = o[a]
        assert np.array_equal(as_bytes(p), o)
    return want


# rows, columns, page_size, share
FORKS = [(1, 1, 1, 1), (4, 9, 16, 4), (7, 33, 13, 3), (40, 20, 8, 8), (130, 70, 4, 2), (300, 200, 16, 10), (33, 3000, 2, 5), (1100, 65, 5, 11)]


@pytest.mark.parametrize("shape", FORKS)
@pytest.mark.parametrize("kind", ["beams", "stay", "free", "wild", "more rows", "fewer rows"])
def test_fork(shape, kind):
    rows, columns, page_size, share = shape
    rng = seed(shape, kind)
    table, length, refs = books(rng, rows, columns, page_size, int(rng.integers(0, 3 * rows + 3)), share)
    parent = np.arange(rows)
    if kind == "beams":
        parent = np.minimum(parent // share * share + rng.integers(0, share, rows), rows - 1)
    elif kind == "free":
        parent[rng.random(rows) < 0.5] = -1
    elif kind == "wild":
        parent = rng.integers(-2, rows + 2, rows)
    elif kind == "more rows":
        parent = rng.integers(0, rows, 2 * rows + 3)
    elif kind == "fewer rows":
        parent = rng.integers(0, rows, rows // 2)
    pools = list(noise(rng, (3, len(refs), 24), torch.bfloat16).unbind(0)) if columns < 1000 else None
    for room in (0, 1, 3 * page_size + 1):
        check_fork(rng, table, length, refs, parent, page_size, room, pools)
    check_fork(rng, table, length, refs, parent, page_size, 0, pools, rng.integers(-1, 2 * page_size, len(parent)))


def test_fork_of_large_books():
    """More pages than one block takes, some of them pinned by others, entries that are no page."""
    rng = seed("large")
    table, length, refs = books(rng, 600, 300, 16, 40000, 6)
    refs[rng.random(len(refs)) < 0.3] += 1
    table[rng.random(table.shape) < 0.01] = -7
    table[0, 0] = len(refs) + 5
    parent = np.arange(600) // 6 * 6 + rng.integers(0, 6, 600)
    parent[rng.random(600) < 0.1] = -1
    for room in (1, 200):
        check_fork(rng, table, length, refs, parent, 16, room)


@pytest.mark.parametrize("pages", [40, 70000])
def test_fork_without_enough_pages_changes_nothing(pages):
    rng = seed("lack", pages)
    table = np.full((4, 50), -1)
    table[:, :3] = np.arange(12).reshape(4, 3)
    length = np.array([40, 48, 33, 48])
    refs = np.ones(pages, np.int64)
    refs[12:15] = 0
    refs[:12] = 1
    parent = np.array([0, 0, 2, 2])                   # rows 1 and 3 go, 6 pages with them
    want = check_fork(rng, table, length, refs, parent, 16, 16 * 5)
    assert want[4][1] > 0 and want[4][2] == 0
    assert check_fork(rng, table, length, refs, parent, 16, 16)[4][1] == 0
    want = check_fork(rng, table, length, refs, parent, 16, 16 * 50)       # more columns than the table has
    assert want[4][1] > 0
    check_fork(rng, table, length, refs, np.array([0, 0, 2, 2, 1, 1, -1]), 16, 16 * 5)


def test_fork_of_no_rows_and_into_none():
    """Everything is freed; rows come out of nothing; single columns; room that is refused for one row is refused for all."""
    rng = seed("none")
    table, length, refs = books(rng, 12, 6, 8, 30, 3)
    want = check_fork(rng, table, length, refs, np.array([], np.int64), 8, 4)
    assert want[4][0] == len(refs)
    empty = (np.zeros((0, 6), np.int64), np.zeros(0, np.int64), np.zeros(40, np.int64))
    check_fork(rng, *empty, np.array([0, -1, 5]), 8, 9)
    check_fork(rng, *empty, np.array([], np.int64), 8, 9)
    check_fork(rng, np.array([[3]]), np.array([0]), np.array([0, 0, 0, 1]), np.array([0, 0, 0]), 2, 2)
    check_fork(rng, table, length, refs, np.arange(12), 8, 0, None, np.where(np.arange(12) == 7, 1 << 30, 0))
    check_fork(rng, table, length, refs, np.arange(12), 8, (1 << 31) - 1)


def test_fork_hands_released_pages_out_again():
    """Every page in use, one sequence freed, another forked onto its pages."""
    rng = seed("again")
    table = np.arange(12).reshape(3, 4)
    length, refs = np.array([25, 32, 32]), np.ones(12, np.int64)
    pools = list(noise(rng, (2, 12, 40), torch.float32).unbind(0))
    want = check_fork(rng, table, length, refs, np.array([0, -1, 0]), 8, 0, pools)
    assert want[4].tolist() == [7, 0, 1, 0] and want[3][0].tolist() == [3, 4]


def test_fork_writes_to_out_and_in_strides():
    rng = seed("out")
    table, length, refs = books(rng, 10, 12, 4, 50, 2)
    wide = torch.full((12, 20), 99, dtype=torch.int32, device="cuda")
    source = torch.full((10, 17), 77, dtype=torch.int32, device="cuda")
    source[:, 2:14] = ints(table)
    parent = np.array([3, 3, 0, 9, 9, 9, -1, 1, 2, 2, 5, 4])
    out = (wide[:, 5:17], torch.empty(12, dtype=torch.int32, device="cuda"), torch.empty(len(refs), dtype=torch.int32, device="cuda"))
    got = C.fork([], source[:, 2:14], ints(length), ints(refs), ints(parent), 4, room=1, out=out)
    want = U.fork(table, length, refs, parent, 4, np.ones(12), 12)
    assert got[0] is out[0] and got[1] is out[1] and got[2] is out[2]
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)
    assert (wide[:, :5] == 99).all() and (wide[:, 17:] == 99).all()


# ---- compact ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("pages", [1, 2, 33, 257, 5000, 70001])
@pytest.mark.parametrize("live", [0.0, 0.02, 0.4, 0.97, 1.0])
@pytest.mark.parametrize("keep", ["live", "half way", "all", "too few"])
def test_compact(pages, live, keep):
    rng = seed(pages, live, keep)
    refs = np.where(rng.random(pages) < live, rng.integers(1, 5, pages), -rng.integers(0, 2, pages))
    table = rng.integers(-2, pages + 2, (9, 31))
    n = int((refs > 0).sum())
    bound = {"live": None, "half way": (n + pages) // 2, "all": pages + 7, "too few": max(n - 1, 0)}[keep]
    pools = list(noise(rng, (2, pages, 20), torch.int16).unbind(0))
    old = [as_bytes(p) for p in pools]
    got = C.compact(pools, ints(table), ints(refs), keep=bound)
    want = U.compact(table, refs, bound)
    for i, what in ((0, "table"), (1, "refs"), (2, "map"), (4, "status")):
        w = want[i] if what != "refs" or not want[4][1] else np.maximum(refs, 0)
        assert np.array_equal(got[i].cpu().numpy(), w), what
    moves = got[3][:len(want[3])].cpu().numpy()
    assert np.array_equal(moves.reshape(-1, 2), np.array(want[3], np.int64).reshape(-1, 2))
    for p, o in zip(pools, old):
        for a, b in want[3]:
            o[b] = o[a]
        assert np.array_equal(as_bytes(p), o)


def test_compact_of_more_tiles_than_blocks():
    rng = seed("tiles")
    pages, pools = 50001, 60
    refs = np.where((np.arange(pages) > 24000) ^ (rng.random(pages) < 0.01), 1, 0)
    table = rng.integers(0, pages, (3, 50))
    whole = noise(rng, (pools, pages, 8), torch.int16)
    old = as_bytes(whole).reshape(pools, pages, -1)
    got = C.compact(list(whole.unbind(0)), ints(table), ints(refs))
    want = U.compact(table, refs, None)
    moves = np.array(want[3], np.int64).reshape(-1, 2)
    assert len(moves) > 20000 and np.array_equal(got[3][:len(moves)].cpu().numpy(), moves)
    old[:, moves[:, 1]] = old[:, moves[:, 0]]
    assert np.array_equal(as_bytes(whole).reshape(pools, pages, -1), old)


# ---- copy ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("page", [1, 3, 16, 585, 1000, 4096, 9000])
@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("other", [False, True])
def test_copy(page, dtype, other):
    rng = seed(page, dtype, other)
    pages, pools = 57, 3
    whole = noise(rng, (pools, pages, page), dtype)
    order = rng.permutation(pages)
    src, dst = order[:20].copy(), order[20:40].copy()
    src[3], dst[5], src[7] = -1, pages, pages + 100
    old = as_bytes(whole)
    to = noise(rng, (pools, pages + 4, page), dtype) if other else whole
    want = as_bytes(to).copy()
    for a, b in zip(src, dst):
        if 0 <= a < pages and 0 <= b < pages + 4 * other:
            want[:, b] = old[:, a]
    got = C.copy(list(whole.unbind(0)), ints(src), ints(dst), to=list(to.unbind(0)) if other else None)
    assert np.array_equal(np.stack([as_bytes(t) for t in got]), want)
    C.copy(list(whole.unbind(0)), ints([]), ints([]))


def test_copy_between_strided_pools():
    """Keys and values of a page side by side; a view that starts off a 16-byte boundary."""
    rng = seed("strided")
    x = noise(rng, (30, 2, 24), torch.bfloat16)
    old = as_bytes(x)
    C.copy([x[:, 0], x[:, 1]], ints([1, 5, 29]), ints([2, 0, 28]))
    want = old.copy()
    want[[2, 0, 28]] = old[[1, 5, 29]]
    assert np.array_equal(as_bytes(x), want)
    flat = noise(rng, (31 * 50 + 3,), torch.uint8)
    y = torch.as_strided(flat, (30, 47), (50, 1), 3)
    z, before = y.clone(), flat.clone()
    C.copy(y, ints([4, 9]), ints([0, 1]))
    z[0], z[1] = z[4].clone(), z[9].clone()
    assert torch.equal(y, z)
    torch.as_strided(before, (30, 47), (50, 1), 3).copy_(z)
    assert torch.equal(flat, before)


# ---- together --------------------------------------------------------------------------------------------------

def test_streams_and_graphs():
    """Two forks captured one after the other with two sets of books, replayed on new parents."""
    rng = seed("graph")
    table, length, refs = books(rng, 24, 20, 4, 400, 4)
    sets = [(ints(table), ints(length), ints(refs)), tuple(torch.empty_like(ints(a)) for a in (table, length, refs))]
    pool = noise(rng, (len(refs), 32), torch.bfloat16)
    first = pool.clone()
    parent = [ints(np.arange(24)), ints(np.arange(24))]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        C.fork(pool, *sets[0], parent[0], 4, room=1, out=sets[1])            # sets the kernels up before the capture
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = C.fork(pool, *sets[0], parent[0], 4, room=1, out=sets[1])
        b = C.fork(pool, *sets[1], parent[1], 4, room=0, out=sets[0])
    books_now, data = (table, length, refs), as_bytes(first)
    for t, v in zip(sets[0], books_now):
        t.copy_(ints(v))
    pool.copy_(first)
    for step in range(3):
        for p in parent:
            p.copy_(ints(np.arange(24) // 4 * 4 + rng.integers(0, 4, 24)))
        graph.replay()
        for p, room, got in ((parent[0], 1, a), (parent[1], 0, b)):
            want = U.fork(*books_now, p.cpu().numpy(), 4, np.full(24, room), 24)
            for g, w in zip(got, want):
                if got is b:
                    assert np.array_equal(g.cpu().numpy(), w)
            assert np.array_equal(got[3].cpu().numpy(), want[3]) and np.array_equal(got[4].cpu().numpy(), want[4])
            for s, d in want[3]:
                if d >= 0:
                    data[d] = data[s]
            books_now = want[:3]
        assert np.array_equal(as_bytes(pool), data)


def test_refusals():
    x = torch.zeros(6, 8, 4, device="cuda")
    parent = ints([0] * 6)
    for kw in (dict(beams=4), dict(beams=0), dict(), dict(beams=65)):
        with pytest.raises(B.NereusError):
            C.reorder(x, parent, **kw)
    big = torch.zeros(7, 8, 4, device="cuda")
    with pytest.raises(B.NereusError):
        C.reorder(big[:6], parent, out=big[1:])                              # overlaps
    with pytest.raises(B.NereusError):
        C.reorder(x, parent, out=big[:6], beams=2)
    for bad in (dict(parent=parent[:5]), dict(parent=parent.long()), dict(length=parent.float()), dict(dim=0), dict(dim=3)):
        with pytest.raises(ValueError):
            C.reorder(x, bad.pop("parent", parent), beams=2, **bad)
    with pytest.raises(ValueError):
        C.reorder(x.transpose(1, 2), parent, beams=2)
    with pytest.raises(ValueError):
        C.reorder([x, x.half()], parent, beams=2)
    with pytest.raises(ValueError):
        C.reorder(x.clone().requires_grad_(), parent, beams=2)
    table, length, refs = ints(np.zeros((3, 4))), ints([1, 2, 3]), ints(np.ones(10))
    pool, parent = torch.zeros(10, 6, device="cuda"), ints([0, 1, 2])
    for kw in (dict(page_size=0), dict(room=-1), dict(out=(table, length.clone(), refs.clone())), dict(out=(table.clone(), length, refs.clone())),
               dict(out=(ints(np.zeros((3, 5))), length.clone(), refs.clone()))):
        with pytest.raises(B.NereusError):
            C.fork(pool, table, length, refs, parent, kw.pop("page_size", 4), **kw)
    for bad in (dict(refs=refs[:9]), dict(length=length[:2]), dict(table=table.long())):
        a = dict(table=table, length=length, refs=refs) | bad
        with pytest.raises(ValueError):
            C.fork(pool, a["table"], a["length"], a["refs"], parent, 4)
    with pytest.raises(ValueError):
        C.compact(pool, table, refs, keep=-2)
    with pytest.raises(B.NereusError):
        C.compact(pool, table, refs, out=(table, refs.clone()))
    with pytest.raises(B.NereusError):
        C.copy(pool, ints([1]), ints([2]), to=torch.zeros(10, 7, device="cuda"))
    with pytest.raises(B.NereusError):
        C.copy(pool[:9], ints([1]), ints([2]), to=pool[1:])
    with pytest.raises(ValueError):
        C.copy(pool, ints([1]), ints([2, 3]))
