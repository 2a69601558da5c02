"""Logits far from zero, as masks and padding leave them (-1e9 to the type's lowest value) or a low temperature makes them:
as whole rows, as all but a few columns, as the vectors that a thread sees first, and as the largest logits of a row.
Against the definitions in 64 bits (tests/logits_util.py, test_gpu_logits_accuracy.py).

Tolerances, derived before the first run.  An element this far from the row's largest adds nothing, and one of equal size
differs from it by at least a unit in its last place, so that the sums are those of the ordinary logits, or of elements that
are equal: a log-sum-exp is off by the sum's relative error (logits_util.sum_error) and its own rounding, 2^-23 relative
with the product by 1 / T; a distillation as in test_gpu_logits_accuracy.py.
"""
import numpy as np
import pytest
import torch

import logits_util as U
from paper_2609_34645_b200 import logits as L
from test_gpu_logits_accuracy import REST, TYPES, definition, rng_of

pytestmark = pytest.mark.gpu
SIZES = [1e6, 1e9, 5e9, 1e10, 1e12, 1e15, 1e18, 1e20, 1e25, 1e29, 1e31, 3e38]
VOCAB = 20011


def rows_with(v, rng):
    """Ordinary logits with v in: all columns; all but 40; the first vectors of every thread; of one thread; the last ones;
    every other column."""
    x = rng.normal(0, 2, (6, VOCAB))
    x[0] = v
    keep = rng.permutation(VOCAB)[:40]
    row = np.full(VOCAB, v)
    row[keep] = x[1, keep]
    x[1] = row
    x[2, :9000] = v
    for layer in range(0, VOCAB, 2048):                   # vector 3 and its partner of every layer, fp32 and bf16
        for vec in (3 * 4, (3 + 256) * 4, 3 * 8, (3 + 256) * 8):
            x[3, layer + vec:layer + vec + 8] = v
    x[4, -9000:] = v
    x[5, ::2] = v
    return torch.as_tensor(x, dtype=torch.float64).float().cuda()


def near_lse(got, x, t):
    ref = torch.logsumexp(x.double() / t, 1)
    tol = U.sum_error(VOCAB) + 4 * U.EPS * 30 / t + 2.0 ** -22 * ref.abs()
    assert torch.isfinite(got).all()
    assert ((got.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("size", SIZES)
def test_log_sum_exp_of_large_logits(size, sign, dtype):
    x = rows_with(sign * size, rng_of("large", size, sign, dtype)).to(TYPES[dtype])
    x = torch.where(torch.isinf(x), torch.full_like(x, sign * torch.finfo(x.dtype).max), x)
    out, token, lse = L.process(x)
    assert torch.equal(out, x) and torch.equal(token.long(), x.float().argmax(1))
    near_lse(lse, x, 1.0)
    for t in (0.5, 1.0, 2.0):
        if size / t > 3e38:
            continue                                       # x / T is not a float
        _, ids, lse = L.teacher_top(x, 5, temperature=t)
        assert torch.equal(ids[:, 0].long(), x.float().argmax(1))
        near_lse(lse, x, t)


@pytest.mark.parametrize("temperature", [1e-9, 1e-6, 1e-3, 2.0 ** -126])
def test_log_sum_exp_at_low_temperatures(temperature):
    """Ordinary logits over a temperature at which x / T is as large as a mask's value."""
    x = torch.as_tensor(rng_of("cold", temperature).normal(0, 2, (3, VOCAB)), dtype=torch.float32, device="cuda")
    if temperature < 1e-30:
        x = x * 0.001                                      # x / T has to be a float
    x[0] = 0.125
    _, _, lse = L.teacher_top(x, 3, temperature=temperature)
    ref = torch.logsumexp(x.double() / temperature, 1)
    assert ((lse.double() - ref).abs() <= U.sum_error(VOCAB) + 2.0 ** -22 * ref.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("divergence,t", [("forward_kl", 1.0), ("forward_kl", 0.5), ("reverse_kl", 2.0), ("js", 1.0)])
@pytest.mark.parametrize("size", SIZES)
def test_distillation_of_masked_students(size, divergence, t, dtype):
    """The teacher names tokens that the mask leaves, and the rest keeps some mass."""
    rng = rng_of("masked", size, divergence, t, dtype)
    x = rows_with(-size, rng)[1:]
    kept = [torch.nonzero(r > -100)[:, 0].cpu().numpy() for r in x]
    ids = torch.as_tensor(np.stack([rng.permutation(k)[:8] for k in kept]).astype(np.int32), device="cuda")
    x = x.to(TYPES[dtype])
    x = torch.where(torch.isinf(x), torch.full_like(x, torch.finfo(x.dtype).min), x)
    y = x.double() + 0.3 * torch.as_tensor(rng.normal(0, 1, x.shape), device="cuda")
    values, lse = y.gather(1, ids.long()).float(), torch.logsumexp(y / t, 1).float()
    args = (x, ids, values, lse, t, divergence, 0.5)
    d, grad, sums, e, m = definition(*args)
    moved, grad_moved = definition(*args, grow=REST)[:2]
    how = {"lse": lse, "divergence": divergence, "temperature": t}
    tol_d = (moved - d).abs() + 2.0 ** -23 * d.abs() + 1e-13
    z = torch.where(grad == 0, 0.0, (x.double() - m).abs() / t)
    last = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol_g = (grad_moved - grad).abs() + (2.0 ** -21 + 2.0 ** -23 * (2 + 2 * z) + last) * grad.abs() + 1e-14
    loss, saved = L.distill_forward(x, ids, values, **how)
    assert ((loss.double() - d).abs() <= tol_d).all()
    assert ((saved[:, :3].double() - sums).abs() <= (REST + 2.0 ** -24) * sums.abs()).all()
    assert ((L.distill_backward(x, ids, values, saved, **how).double() - grad).abs() <= tol_g).all()
    loss, got = L.distill_step(x, ids, values, **how)
    assert ((loss.double() - d).abs() <= tol_d).all()
    assert ((got.double() - grad).abs() <= tol_g).all()
