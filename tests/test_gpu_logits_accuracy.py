"""How exact the distillation is where a 32-bit evaluation of its formulas loses its digits: students near their teacher,
teachers that leave nearly nothing to the rest.  Against the definition in 64 bits.

Tolerances, derived before the first run.  Everything a row has once per entry is worked out in 64 bits, so only three
things are left, and each is followed through the definition itself:
  * the sum over the rest, in fp32: the exponential's 2^-22 (the bound of its instruction), once for all elements, and as
    much again for the roundings of the partial sums, which are independent: REST = 2^-21.  What that does to a loss or a
    gradient is the definition's difference between the rest's sum and that sum times 1 + REST.
  * an element of the rest in the gradient: two exponentials' 2^-22 each, three roundings, and the rounding of the exponent
    (x - m) / T and of its factor, 2^-24 of it each: EACH(z) = 2^-21 + 2^-23 (2 + 2 |z|), relative.
  * the rounding of what is written: rounding keeps order, so a written value lies between the type's roundings of the
    exact one less and plus its tolerance.
"""
import zlib

import numpy as np
import pytest
import torch

from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu
REST = 2.0 ** -21
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
RMS = {"bf16": 2.0 ** -8.8, "fp32": 2.0 ** -24.8}         # of a rounding: half a unit in the last place over sqrt(3)

# divergence, whether the rest is a group, temperature, beta
HOW = [("forward_kl", True, 1.0, 0.5), ("forward_kl", False, 0.7, 0.5), ("reverse_kl", True, 1.0, 0.5),
       ("reverse_kl", True, 2.0, 0.5), ("js", True, 0.7, 0.3), ("js", True, 1.0, 0.5), ("forward_kl", True, 0.7, 0.5)]


def rng_of(*key):
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def teachers(rng, vocab, k, t, what):
    """Rows (x, ids, values, lse): what = (P_rest, how far the student is from the teacher, the size of the logits)."""
    x, ids, values, lse = [], [], [], []
    for p_rest, far, level in what:
        at = rng.permutation(vocab)[:k]
        logp = np.sort(rng.normal(0, 2.0, k))[::-1]
        logp += np.log1p(-p_rest) - np.log(np.exp(logp).sum())
        row = rng.normal(0, 1.6, vocab)
        rest = np.ones(vocab, bool)
        rest[at] = False
        # the rest gets P_rest times a factor near one
        row += (np.log(p_rest) + far * rng.normal() - np.log(np.exp(row[rest] / t).sum())) * t
        row[at] = (logp + far * rng.normal(0, 1, k)) * t
        x.append(row + 0.37 * level)
        ids.append(at)
        values.append(logp * t + level * t)
        lse.append(level)
    as32 = lambda a: torch.as_tensor(np.array(a), dtype=torch.float32, device="cuda")              # noqa: E731
    return as32(x), torch.as_tensor(np.array(ids), dtype=torch.int32, device="cuda"), as32(values), as32(lse)


def definition(x, ids, values, lse, t, divergence, beta, grow=0.0):
    """(D, gradient, sums) in 64 bits; the sum over the rest is taken 1 + grow times as large."""
    x, ids, values = x.double(), ids.long(), values.double()
    m = x.amax(1, keepdim=True)
    e = torch.exp((x - m) / t)
    of_entries = e.gather(1, ids)
    rest = e.scatter(1, ids, 0.0).sum(1, keepdim=True) * (1 + grow)
    total = rest + of_entries.sum(1, keepdim=True)
    q = torch.cat([of_entries, rest], 1) / total
    log_q = torch.cat([(x.gather(1, ids) - m) / t, torch.log(rest)], 1) - torch.log(total)
    if lse is None:
        log_p = torch.cat([torch.log_softmax(values / t, 1), torch.full_like(m, -np.inf)], 1)
        p = torch.exp(log_p)
    else:
        p = torch.exp(values / t - lse.double()[:, None])
        p_rest = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        p = torch.cat([p, p_rest], 1)
        log_p = torch.cat([values / t - lse.double()[:, None], torch.log(p_rest)], 1)
    if divergence == "forward_kl":
        d = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
        qf = -p
    elif divergence == "reverse_kl":
        log_p[:, -1] = log_p[:, -1].clamp(min=-24 * np.log(2.0))
        qf = q * (log_q - log_p)
        d = qf.sum(1)
    else:
        log_m = torch.log(beta * p + (1 - beta) * q)
        qf = q * (1 - beta) * (log_q - log_m)
        d = (qf + torch.where(p > 0, beta * p * (log_p - log_m), 0.0)).sum(1)
    slope = (qf - q * qf.sum(1, keepdim=True)) / t                       # of a whole group
    grad = (e * (slope[:, -1:] / rest) * (1 + grow)).scatter(1, ids, slope[:, :-1])
    return d, grad, torch.cat([m, total, rest], 1), e, m


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,k", [(1000, 7), (50257, 64), (128256, 200)])
@pytest.mark.parametrize("divergence,with_rest,t,beta", HOW)
def test_near_students_and_small_rests(divergence, with_rest, t, beta, vocab, k, dtype):
    rng = rng_of(divergence, with_rest, t, beta, vocab, dtype)
    what = [(p, far, 0.0) for p in (2.0 ** -22, 2.0 ** -19, 2.0 ** -14, 2.0 ** -9, 0.25) for far in (0.005, 0.05, 1.0)]
    what += [(p, far, 17.3) for p in (2.0 ** -12, 2.0 ** -9, 0.25) for far in (0.005, 0.05, 1.0)]
    if divergence == "reverse_kl":
        what += [(2.0 ** -26, far, 0.0) for far in (0.05, 1.0)]
    x, ids, values, lse = teachers(rng, vocab, k, t, what)
    x = x.to(TYPES[dtype])
    args = (x, ids, values, lse if with_rest else None, t, divergence, beta)
    d, grad, sums, e, m = definition(*args)
    d_moved, grad_moved, _, _, _ = definition(*args, grow=REST)
    how = {"lse": lse if with_rest else None, "divergence": divergence, "temperature": t, "beta": beta}
    up = torch.as_tensor(rng.uniform(0.5, 2, len(what)), dtype=torch.float32, device="cuda")

    tol_d = (d_moved - d).abs() + 1e-13
    z = ((x.double() - m) / t).abs()
    tol_g = (grad_moved - grad).abs() + (2.0 ** -21 + 2.0 ** -23 * (2 + 2 * z)) * grad.abs() + 1e-14

    def near(got, want, tol, name):
        low, high = ((want + s * tol).to(got.dtype) for s in (-1, 1))
        off = ((got.double() - want).abs() / tol).max().item()
        assert ((low <= got) & (got <= high)).all(), f"{name}: {off:.3g} times the tolerance, rounding included"

    loss, saved = L.distill_forward(x, ids, values, **how)
    near(loss, d, tol_d, "forward's loss")
    near(saved[:, :3], sums, REST * sums.abs() + 1e-30, "saved sums")
    near(saved[:, 3], d, tol_d, "saved divergence")
    # where the loss is worth anything, the tolerance above is a few millionths of it
    worth = d >= 1e-3
    assert (tol_d[worth] <= 1e-5 * d[worth]).all()
    step_loss, step_grad = L.distill_step(x, ids, values, **how)
    near(step_loss, d, tol_d, "step's loss")
    near(step_grad, grad, tol_g, "step's gradient")
    back = L.distill_backward(x, ids, values, saved, grad_loss=up, **how)
    near(back, grad * up.double()[:, None], tol_g * up.double()[:, None], "backward's gradient")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("divergence,with_rest,t,beta", HOW)
def test_gradients_of_large_rows_sum_to_zero(divergence, with_rest, t, beta, dtype):
    """Adding one number to all logits changes nothing, so a row's gradient sums to zero: up to the tolerance of each
    element, which for independent roundings adds up by squares."""
    rng = rng_of("sum", divergence, with_rest, t, dtype)
    x, ids, values, lse = teachers(rng, 152064, 128, t, [(p, far, 0.0) for p in (2.0 ** -9, 0.1, 0.5) for far in (0.1, 1.0)])
    x = x.to(TYPES[dtype])
    _, grad = L.distill_step(x, ids, values, lse=lse if with_rest else None, divergence=divergence, temperature=t, beta=beta)
    g = grad.double()
    systematic = 2.0 ** -21 + 2.0 ** -22 * 30                # the exponential's and its factor's, at |x - m| / T up to 30
    assert (g.sum(1).abs() <= systematic * g.abs().sum(1) + 4 * RMS[dtype] * g.square().sum(1).sqrt()).all()
