"""A beam search's selection against its definition in 64 bits.

Tolerances, derived before the first run.  A total is score + x - lse, worked out in 64 bits from a sum of exponentials in
fp32: sum_error(V) relative (tests/logits_util.py), so that much absolute in the logarithm, and one rounding to fp32 of the
result, 2^-24 relative.  Which hypotheses come out, and in which order, is equal: where two of them differ by less than what
the sums can be off (2e-6 here; equal ones not among them) either order is right.
"""
import numpy as np
import pytest
import torch

import logits_util as U
from paper_2609_34645_b200 import binding as B
from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu
INF = float("inf")
NEAR = 2e-6

# requests, beams, vocab, tp, padded, k
SHAPES = [(1, 1, 1, 1, False, 1), (1, 1, 1, 1, False, 5), (2, 3, 7, 1, False, 6), (1, 4, 129, 2, True, 8), (3, 5, 1000, 4, False, 10),
          (2, 2, 4099, 1, False, 4), (3, 4, 50257, 4, True, 8), (1, 8, 32064, 8, False, 16), (1, 1, 128256, 1, False, 128),
          (5, 3, 300, 64, True, 3), (1, 64, 2051, 1, False, 128), (2, 64, 129, 1, False, 64), (20, 6, 8192, 2, False, 12),
          (1, 4, 128256, 1, False, 8), (2, 3, 152064, 2, False, 6), (1, 32, 20011, 1, False, 64)]
LAYOUTS = ["shards", "columns", "odd"]


def definition(x, score, k, beams, ended=None, norm=None):
    """(totals, ranks) of all hypotheses of every request in 64 bits, [requests, beams * vocab]; -inf: not offered."""
    rows, vocab = x.shape
    with np.errstate(all="ignore"):
        lse = U.log_sum_exp(x)
        total = score.astype(np.float64)[:, None] + x - lse[:, None]
        total[~np.isfinite(lse)] = -INF
        if ended is not None:
            for r in np.flatnonzero((ended >= 0) & (ended < vocab)):
                total[r] = -INF
                total[r, ended[r]] = score[r]
        dead = ~np.isfinite(score)
        rank = total
        if norm is not None:
            n = norm.astype(np.float64)
            dead |= ~((n > 0) & np.isfinite(n))
            rank = total / n[:, None]
        total, rank = total.copy(), rank.copy()
        for v in (total, rank):
            v[dead] = -INF
            v[np.isnan(v)] = -INF
    return total.reshape(-1, beams * vocab), rank.reshape(-1, beams * vocab)


def settled(beam, beams):
    """Places of hypotheses in rank order (beam -1: none) when what goes on from a row first is put at its place."""
    place, lead = np.full(len(beam), -1), {}
    for j, b in enumerate(beam):
        if b >= 0 and b not in lead:
            lead[b] = j
            place[j] = b
    vacant = [b for b in range(beams) if b not in lead]
    for j in range(len(beam)):
        if place[j] < 0:
            place[j] = vacant.pop(0)
    return place


def check(view, x, score, k, beams, ended=None, norm=None, settle=False):
    dev = lambda a, t: None if a is None else torch.as_tensor(a).to("cuda", t)                     # noqa: E731
    got = L.beam_select(view.arg(), dev(score, torch.float32), k, beams=beams, vocab=view.vocab, ended=dev(ended, torch.int32),
                        norm=dev(norm, torch.float32), settle=settle)
    value, parent, token = (t.cpu().numpy() for t in got)
    total, rank = definition(x, score, k, beams, ended, norm)
    requests, vocab = len(total), view.vocab
    assert value.shape == parent.shape == token.shape == (requests, k)
    tol = U.sum_error(vocab)
    for g in range(requests):
        want = np.argsort(-rank[g], kind="stable")[:k]
        want = np.concatenate([want[rank[g][want] > -INF], np.full(k, -1)])[:k].astype(np.int64)
        if settle:
            place = settled([w // vocab if w >= 0 else -1 for w in want], beams)
            order = place                            # the j-th by rank is at place[j]
        else:
            order = np.arange(k)
        here = np.where(token[g] >= 0, (parent[g] - g * beams) * vocab + token[g], -1)[order]
        assert ((parent[g] >= 0) == (token[g] >= 0)).all()
        for j in range(k):
            a, b = here[j], want[j]
            if a != b:
                assert a >= 0 and b >= 0, (g, j, a, b)
                gap = abs(rank[g][a] - rank[g][b])
                assert 0 < gap < NEAR, (g, j, a, b, gap)
        assert len(set(here[here >= 0])) == (here >= 0).sum()
        expect = np.where(here >= 0, total[g][np.maximum(here, 0)], -INF)
        off = np.abs(value[g][order].astype(np.float64)[here >= 0] - expect[here >= 0])
        assert (off <= tol + U.EPS * np.abs(expect[here >= 0])).all(), (g, off)
        assert (value[g][order][here < 0] == -INF).all()
    return value, parent, token


def logits(rng, rows, vocab, dtype):
    x = rng.normal(0, 2, (rows, vocab))
    for r in range(rows):
        x[r, rng.integers(0, vocab, 6)] += rng.uniform(3, 8, 6)
    return U.rounded(x, dtype)


def seed(*key):
    import zlib
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_against_the_definition(shape, dtype, layout):
    requests, beams, vocab, tp, padded, k = shape
    rng = seed(shape, dtype, layout)
    rows = requests * beams
    x = logits(rng, rows, vocab, dtype)
    score = rng.uniform(-20, 0, rows).astype(np.float32)
    view = U.View(rows, vocab, tp, dtype, layout, padded).put(torch.as_tensor(x))
    check(view, x, score, k, beams)
    ended = np.where(rng.random(rows) < 0.3, rng.integers(0, vocab, rows), -1).astype(np.int32)
    score[rng.random(rows) < 0.2] = -INF
    norm = rng.uniform(0.5, 3, rows).astype(np.float32)
    check(view, x, score, k, beams, ended, norm)
    check(view, x, score, beams, beams, ended, norm, settle=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["equal", "masked", "lowest", "few", "none", "two values", "far", "ties"])
@pytest.mark.parametrize("shape", [(2, 4, 50257, 8), (3, 1, 8200, 128), (2, 64, 1030, 128), (1, 5, 128256, 10)])
def test_rows_of_few_values(shape, dtype, kind):
    """Rows that a mask has left little of, rows of equal elements: ties go to the lowest beam and token."""
    requests, beams, vocab, k = shape
    rng = seed(shape, dtype, kind)
    rows = requests * beams
    low = float(torch.finfo(U.TYPES[dtype]).min)
    x = logits(rng, rows, vocab, dtype)
    keep = np.zeros((rows, vocab), bool)
    for r in range(rows):
        keep[r, rng.integers(0, vocab, 3)] = True
    if kind == "equal":
        x[:] = 1.5
    elif kind == "masked":
        x[~keep] = -1e10
        x = U.rounded(x, dtype)
    elif kind == "lowest":
        x[~keep] = low
    elif kind == "few":
        x[~keep] = -INF
    elif kind == "none":
        x[1:] = -INF
    elif kind == "two values":
        x = np.where(rng.random((rows, vocab)) < 0.1, 2.0, 1.0)
    elif kind == "far":
        x = U.rounded(x + rng.choice([-1e4, 3e5, 0], (rows, 1)), dtype)
    elif kind == "ties":
        x = np.round(x / 2) * 2
    score = np.round(rng.uniform(-20, 0, rows)).astype(np.float32)
    view = U.View(rows, vocab, 1, dtype, "columns").put(torch.as_tensor(x))
    check(view, x, score, k, beams)
    check(view, x, score, beams, beams, norm=np.full(rows, 2.0, np.float32), settle=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_equal_beams_go_by_their_row(dtype):
    """The first step of a search that forgot to give all beams but one a score of -inf: every beam offers the same."""
    rng = seed("equal", dtype)
    x = np.repeat(logits(rng, 3, 32768, dtype), 8, axis=0)
    view = U.View(24, 32768, 1, dtype, "columns").put(torch.as_tensor(x))
    value, parent, token = check(view, x, np.zeros(24, np.float32), 16, 8)
    assert (parent % 8 == np.tile(np.arange(8), 2)).all() and (token[:, :8] == token[:, :1]).all()
    _, parent, _ = check(view, x, np.where(np.arange(24) % 8 == 0, 0, -INF).astype(np.float32), 8, 8)
    assert (parent % 8 == 0).all()


def test_what_offers_nothing():
    """Scores and norms that are no numbers, rows with NaN or +inf, rows of -inf, ended beams among them."""
    rng = seed("nothing")
    beams, vocab = 12, 3001
    x = logits(rng, 2 * beams, vocab, "fp32")
    score = rng.uniform(-5, 0, 2 * beams).astype(np.float32)
    norm = np.ones(2 * beams, np.float32)
    ended = np.full(2 * beams, -1, np.int32)
    score[[0, 1, 2]] = INF, -INF, np.nan
    norm[[3, 4, 5, 6]] = 0.0, -1.0, np.nan, INF
    x[7, 77] = np.nan
    x[8, 88] = INF
    x[9] = -INF
    x[10], ended[10] = np.nan, 17                     # ended: its row is not read
    score[11], ended[11] = -INF, 3
    score[12:] = -INF                                 # a request with nothing at all
    ended[13] = vocab                                 # outside: goes on
    view = U.View(2 * beams, vocab, 1, "fp32", "shards").put(torch.as_tensor(x))
    value, parent, token = check(view, x, score, 20, beams, ended, norm)
    assert (parent[0] == [10] + [-1] * 19).all() and token[0, 0] == 17 and (parent[1] == -1).all()
    score[14], ended[13], score[13] = -1.0, 5, -2.0
    check(view, x, score, 12, beams, ended, norm, settle=True)


def test_the_same_bits_in_any_batch():
    """A request's results do not depend on the others', nor on where it stands, as long as its rows start alike."""
    rng = seed("batch")
    x = torch.as_tensor(logits(rng, 60, 16384, "bf16"))
    score = torch.as_tensor(rng.uniform(-9, 0, 60).astype(np.float32)).cuda()
    whole = x.bfloat16().cuda()
    value, parent, token = L.beam_select(whole, score, 10, beams=5)
    for g in (0, 3, 11):
        cut = slice(5 * g, 5 * g + 5)
        v, p, t = L.beam_select(whole[cut].clone(), score[cut].clone(), 10, beams=5)
        assert torch.equal(v[0], value[g]) and torch.equal(p[0] + 5 * g, parent[g]) and torch.equal(t[0], token[g])


def test_captured_and_on_another_stream():
    rng = seed("graph")
    x = torch.as_tensor(logits(rng, 8, 50257, "bf16")).bfloat16().cuda()
    score = torch.zeros(8, device="cuda")
    want = L.beam_select(x, score, 8, beams=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = L.beam_select(x, score, 8, beams=4)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = L.beam_select(x, score, 8, beams=4)
    y = torch.as_tensor(logits(rng, 8, 50257, "bf16")).bfloat16().cuda()
    x0 = x.clone()
    x.copy_(y)
    graph.replay()
    other = L.beam_select(y, score, 8, beams=4)
    assert all(torch.equal(a, b) for a, b in zip(out, other))
    x.copy_(x0)
    graph.replay()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, out, again))


def test_no_rows_and_refusals():
    x, score = torch.zeros(0, 100, device="cuda"), torch.zeros(0, device="cuda")
    assert [t.shape for t in L.beam_select(x, score, 4, beams=2)] == [(0, 4)] * 3
    x, score = torch.zeros(6, 100, device="cuda"), torch.zeros(6, device="cuda")
    for wrong in (dict(beams=4, k=4), dict(beams=0, k=4), dict(beams=65, k=4), dict(beams=2, k=0), dict(beams=2, k=129),
                  dict(beams=2, k=4, settle=True)):
        with pytest.raises(B.NereusError):
            L.beam_select(x, score, wrong.pop("k"), **wrong)
    for wrong in (dict(score=score[:5]), dict(score=score.double()), dict(ended=score), dict(norm=score.int()), dict(score=score.cpu())):
        with pytest.raises(ValueError):
            L.beam_select(x, wrong.pop("score", score), 4, beams=2, **wrong)
    with pytest.raises(ValueError):
        L.beam_select(x.half(), score, 4, beams=2)


@pytest.mark.parametrize("vocab, rows, beams", [(128256, 5200, 4), (700, 9000, 3)])
def test_more_rows_than_are_listed(vocab, rows, beams):
    """More rows than the summing blocks list, and more layers to a block than its table holds; most of them are not read."""
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(rows, vocab, generator=gen, device="cuda").mul_(2).bfloat16()
    score = -torch.rand(rows, generator=gen, device="cuda")
    score[torch.rand(rows, generator=gen, device="cuda") < 0.3] = -INF
    k = 2 * beams
    value, parent, token = L.beam_select(x, score, k, beams=beams)
    for a in range(0, rows, 60 * beams):
        b = min(rows, a + 60 * beams)
        total = x[a:b].double().log_softmax(1) + score[a:b].double()[:, None]
        want = total.view(-1, beams * vocab).topk(k, dim=1).values
        g = slice(a // beams, b // beams)
        live = want > -INF
        assert torch.equal(live, parent[g] >= 0)
        tol = U.sum_error(vocab) + U.EPS * want.abs()
        assert ((value[g].double() - want).abs()[live] <= tol[live]).all()
        at = (parent[g].clamp(min=a).long() - a) * vocab + token[g].clamp(min=0).long()
        got = total.view(-1)[at]
        assert ((got - want).abs()[live] < NEAR).all()                      # what was picked is worth what it has to be
        assert all(len(set(r)) == len(r) for r in at[live.all(1)].tolist())
        assert (value[g][~live] == -INF).all()


def test_norms_at_the_ends_of_their_range():
    """Quotients beyond fp32 and next to 0: the order is theirs in 64 bits."""
    rng = seed("norms")
    x = logits(rng, 8, 3000, "fp32")
    view = U.View(8, 3000, 1, "fp32", "columns").put(torch.as_tensor(x))
    for norm in (1e-44, 1e-39, 1e-30, 1e30, 3e38):
        n = np.full(8, norm, np.float32)
        check(view, x, rng.uniform(-9, 0, 8).astype(np.float32), 8, 4, norm=n)
        check(view, x, rng.uniform(20, 40, 8).astype(np.float32), 8, 4, norm=n)
