"""Selections whose quotients, norms or offsets lie at or beyond the ends of fp32: what is offered, and its order, is by the totals
and quotients in 64 bits.

Tolerances as in tests/test_gpu_beam.py: a row's totals are off together by the error of its sum, so that hypotheses of two rows
whose totals lie closer than that may change places; of totals t and u at norms n and m that is |t / n - u / m| below
error / n + error / m.  Totals themselves: that error and one rounding to fp32."""
import numpy as np
import pytest
import torch

import logits_util as U
from test_gpu_beam import definition, seed
from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu
INF = float("inf")


def check(x, score, norm, k, beams):
    rows, vocab = x.shape
    view = U.View(rows, vocab, 1, "fp32", "columns").put(torch.as_tensor(x))
    got = L.beam_select(view.arg(), torch.as_tensor(score).cuda(), k, beams=beams, norm=torch.as_tensor(norm).cuda())
    value, parent, token = (t.cpu().numpy() for t in got)
    total, rank = definition(x, score, k, beams, None, norm)
    tol = U.sum_error(vocab)
    for g in range(rows // beams):
        want = np.argsort(-rank[g], kind="stable")[:k]
        assert (rank[g][want] > -INF).all() and (parent[g] >= 0).all()
        here = (parent[g] - g * beams) * vocab + token[g]
        assert len(set(here.tolist())) == k
        per = norm[g * beams:(g + 1) * beams].astype(np.float64)
        for b in range(beams):                                           # a row's own order has no error
            own = here[here // vocab == b]
            assert np.array_equal(own, b * vocab + np.argsort(-rank[g][b * vocab:(b + 1) * vocab], kind="stable")[:len(own)])
        for a, b in zip(here, want):
            assert abs(rank[g][a] - rank[g][b]) <= tol / per[a // vocab] + tol / per[b // vocab]
        off = np.abs(value[g].astype(np.float64) - total[g][here])
        assert (off <= tol + U.EPS * np.abs(total[g][here])).all()


def near(rng, rows, vocab, target):
    """Logits and scores whose totals all lie within 0.1 of `target`, no two of a row alike."""
    x = U.rounded(rng.permutation(rows * vocab).reshape(rows, vocab) * (0.1 / (rows * vocab)), "fp32")
    return x, (target + U.log_sum_exp(x) - 0.05).astype(np.float32)


@pytest.mark.parametrize("target", [0.0, 0.1, 1.0, -0.1, -1.0])
@pytest.mark.parametrize("norm", [1e-45, 1e-44, 1e-39, 2.0 ** -127, 2.9e-39, 2.0 ** -126, 1e-30, 1e30, 1e36, 1e38, 3e38])
def test_norms_whose_inverse_or_quotients_leave_fp32(norm, target):
    rng = seed(norm, target)
    x, score = near(rng, 8, 3000, target)
    check(x, score, np.full(8, norm, np.float32), 8, 4)
    check(x, score, np.full(8, norm, np.float32), 70, 8)


@pytest.mark.parametrize("target", [0.0, 0.1, -0.1, 30.0, -30.0])
def test_norms_of_all_sizes_in_one_request(target):
    rng = seed("mixed", target)
    x, score = near(rng, 16, 3000, target)
    for some in ((1e-44, 1.0), (1e-39, 1e-37, 3.0, 1e38), (3e38, 1e20), (1e-45, 3e38)):
        check(x, score, np.resize(np.array(some, np.float32), 16), 12, 8)
        check(x, score, np.repeat(np.array(some, np.float32), 16 // len(some)), 12, 16)


def test_offsets_beyond_fp32():
    """A row far below 0 at a score as far above it: what every token adds to its logit is no fp32."""
    vocab = 3000
    x = np.zeros((4, vocab))
    x[0] = U.rounded(-3e38 - 1e32 * np.arange(vocab), "fp32")
    x[2] = U.rounded(3e38 - 1e35 * np.arange(vocab), "fp32")
    score = np.array([3e38, 3.2e38, -3e38, -3.3e38], np.float32)
    for k in (4, 9):
        check(x, score, np.ones(4, np.float32), k, 2)
        check(x, score, np.array([2, 1, 1, 1], np.float32), k, 2)
