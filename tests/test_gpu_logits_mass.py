"""Teachers whose probabilities do not sum to one: a log-sum-exp of another temperature, or one that is off, so that the
entries alone have more than all mass; and entries that are all of the vocabulary.  The gradient is that of the loss that is
returned with it, by the formula (-P/Q in the forward KL) and by differences of the 64-bit loss.

Tolerances as in test_gpu_logits_accuracy.py; central differences with h = 1e-4 are off by h^2 / 6 of the third derivative,
which is below the mass (at most 4) over T^3, and by the 64-bit loss's rounding over h: together below 1e-7."""
import numpy as np
import pytest
import torch

from paper_2609_34645_b200 import logits as L
from test_gpu_logits_accuracy import HOW, REST, definition, rng_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("all_tokens", [False, True])
@pytest.mark.parametrize("divergence,t,beta", sorted({(d, t, b) for d, with_rest, t, b in HOW if with_rest}))
def test_gradient_of_teachers_with_another_mass(divergence, t, beta, all_tokens):
    rng = rng_of("mass", divergence, t, beta, all_tokens)
    vocab = 40
    k = vocab if all_tokens else 12
    shift = np.array([-1.2, -0.5, -0.01, 0.0, 0.4])          # the entries' mass: 3.3, 1.6, 1.01, 1, 0.67 of what it should be
    as32 = lambda a: torch.as_tensor(np.array(a), dtype=torch.float32, device="cuda")              # noqa: E731
    x = as32(rng.normal(0, 2, (len(shift), vocab)))
    y = x.double().cpu().numpy() + rng.normal(0, 0.5, x.shape)
    ids = np.argsort(-y, axis=1)[:, :k]
    values = as32(np.take_along_axis(y, ids, 1))
    lse = as32(np.log(np.exp(np.take_along_axis(y, ids, 1) / t).sum(1)) + shift)
    ids = torch.as_tensor(ids.astype(np.int32), device="cuda")

    def loss_of(z):
        """Every token an entry: the rest has no mass on either side and takes no part."""
        if not all_tokens:
            return definition(z, ids, values, lse, t, divergence, beta)[0]
        log_q = torch.log_softmax(z / t, 1).gather(1, ids.long())
        log_p = values.double() / t - lse.double()[:, None]
        p, q = log_p.exp(), log_q.exp()
        if divergence == "forward_kl":
            return (p * (log_p - log_q)).sum(1)
        if divergence == "reverse_kl":
            return (q * (log_q - log_p)).sum(1)
        log_m = torch.log(beta * p + (1 - beta) * q)
        return (beta * p * (log_p - log_m) + (1 - beta) * q * (log_q - log_m)).sum(1)

    z = x.double().requires_grad_()
    loss_of(z).sum().backward()
    want, d = z.grad, loss_of(x.double())
    how = {"lse": lse, "divergence": divergence, "temperature": t, "beta": beta}
    loss, grad = L.distill_step(x, ids, values, **how)
    _, saved = L.distill_forward(x, ids, values, **how)
    back = L.distill_backward(x, ids, values, saved, **how)
    # of a sum over the rest that is off by REST: at most that of every token's own slope, and of the mass
    tol = 8 * REST * (1 + want.abs().max()) / t
    assert ((loss.double() - d).abs() <= tol).all()
    for got in (grad, back):
        assert ((got.double() - want).abs() <= tol).all()
        for v in range(0, vocab, 7):
            up, down = x.double(), x.double()
            up[:, v] += 1e-4
            down[:, v] -= 1e-4
            diff = (loss_of(up) - loss_of(down)) / 2e-4
            assert ((got[:, v].double() - diff).abs() <= tol + 1e-7).all()
