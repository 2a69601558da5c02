"""A rest that lies far below the entries, in the logits or by a low temperature: its sum in units of the largest logit's
exponential is no fp32 from 87 on, and with a weight the gradient's factor, P_rest over that sum, was none before that.
Tolerances as in test_gpu_logits_accuracy.py: 64 bits hold everything here down to 700."""
import numpy as np
import pytest
import torch

from paper_2609_34645_b200 import logits as L
from test_gpu_logits_accuracy import REST, definition, rng_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("divergence", ["forward_kl", "reverse_kl", "js"])
@pytest.mark.parametrize("t,weight", [(1.0, 1.0), (1.0, 1000.0), (0.05, 50.0), (4.0, 1e-3)])
@pytest.mark.parametrize("gap", [30, 60, 80, 85, 88, 95, 110, 200, 700])
def test_rest_far_below_the_entries(gap, t, weight, divergence):
    rng = rng_of("rest", gap, t, weight, divergence)
    rows, vocab, k = 4, 5003, 6
    x = rng.normal(0, 1, (rows, vocab)) * t
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)])
    x[np.arange(rows)[:, None], ids] += (gap + 8) * t
    x = torch.as_tensor(x, dtype=torch.float32, device="cuda")
    ids = torch.as_tensor(ids.astype(np.int32), device="cuda")
    values = torch.as_tensor(rng.normal(0, 1, (rows, k)) * t, dtype=torch.float32, device="cuda")
    lse = (torch.logsumexp(values.double() / t, 1) + torch.tensor([0.0, 0.05, 0.5, 2.0], device="cuda")).float()
    args = (x, ids, values, lse, t, divergence, 0.5)
    d, grad, sums, e, m = definition(*args)
    moved, grad_moved = definition(*args, grow=REST)[:2]
    w = torch.full((rows,), weight, device="cuda")
    how = {"lse": lse, "divergence": divergence, "temperature": t, "weight": w}
    w = w.double()
    # the gradient's exponentials start at the rest's own largest: 12 T or less from each of its elements
    tol_d = ((moved - d).abs() + 2.0 ** -23 * d.abs() + 1e-13) * w
    tol_g = ((grad_moved - grad).abs() + (2.0 ** -21 + 2.0 ** -23 * (2 + 2 * 24) + 2.0 ** -24) * grad.abs()) * w[:, None] + 2.0 ** -149
    tol_g += 1e-15 * w[:, None] / t
    loss, saved = L.distill_forward(x, ids, values, **how)
    assert ((loss.double() - d * w).abs() <= tol_d).all()
    loss, got = L.distill_step(x, ids, values, **how)
    assert ((loss.double() - d * w).abs() <= tol_d).all()
    assert torch.isfinite(got).all() and ((got.double() - grad * w[:, None]).abs() <= tol_g).all()
    got = L.distill_backward(x, ids, values, saved, **how)
    assert torch.isfinite(got).all()
    if gap <= 80:                                              # S_rest is a normal number
        assert ((got.double() - grad * w[:, None]).abs() <= tol_g).all()
