"""A vocabulary that does not divide, cut without padding: the last shard is narrower than the others, as
``x.split(w, dim=1)`` gives it.  Results equal the uncut tensor's: nothing but the order of fp32 sums may differ, which
moves a log-sum-exp or a loss by the sum's error (logits_util.sum_error) and a gradient by as much, relative."""
import pytest
import torch

import logits_util as U
from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu


def _split(x, w):
    return list(x.split(w, dim=1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,w", [(1, 10, 4), (3, 50257, 12565), (5, 1001, 500), (4, 4099, 4096), (2, 27, 10)])
def test_default_outputs_of_a_narrower_last_shard(rows, vocab, w, dtype):
    gen = torch.Generator("cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, device="cuda", generator=gen).to(dtype)
    tol = U.sum_error(vocab) + 8 * U.EPS * 16
    near = lambda a, b: bool(((a.float() - b.float()).abs() <= tol * (1 + b.float().abs())).all())           # noqa: E731
    out, token, lse = L.process(_split(x, w), vocab=vocab)
    assert [o.shape for o in out] == [s.shape for s in _split(x, w)] and out[0].dtype == dtype
    assert torch.equal(torch.cat(out, 1), x) and torch.equal(token, L.process(x)[1]) and near(lse, L.process(x)[2])
    out, _, _ = L.process(_split(x, w), vocab=vocab, out_dtype=torch.float32)
    assert torch.equal(torch.cat(out, 1), x.float())

    values, ids, lse = L.teacher_top((x.float() + torch.randn(x.shape, device="cuda", generator=gen)).to(dtype), 3)
    loss, grad = L.distill_step(x, ids, values, lse=lse)
    got_loss, got = L.distill_step(_split(x, w), ids, values, vocab=vocab, lse=lse)
    rel = 2.0 ** -7 if dtype == torch.bfloat16 else 8 * tol
    assert near(got_loss, loss) and ((torch.cat(got, 1).float() - grad.float()).abs() <= rel * grad.float().abs() + 1e-7).all()
    loss, saved = L.distill_forward(_split(x, w), ids, values, vocab=vocab, lse=lse)
    got = L.distill_backward(_split(x, w), ids, values, saved, vocab=vocab, lse=lse)
    assert near(loss, got_loss) and ((torch.cat(got, 1).float() - grad.float()).abs() <= rel * grad.float().abs() + 1e-7).all()

    y = x.clone().requires_grad_()
    L.distill_loss(_split(y, w), ids, values, vocab=vocab, lse=lse).sum().backward()
    assert ((y.grad.float() - grad.float()).abs() <= rel * grad.float().abs() + 1e-7).all()


def test_a_narrower_last_shard_that_is_padded_too():
    """27 tokens over shards of 10, 10 and 8 columns: the last column is padding and its gradient is zero."""
    whole = torch.randn(6, 28, device="cuda")
    whole[:, 27] = float("nan")
    y = whole.clone().requires_grad_()
    values, ids, lse = L.teacher_top(whole[:, :27].contiguous(), 3)
    L.distill_loss(_split(y, 10), ids, values, vocab=27, lse=lse).sum().backward()
    assert torch.isfinite(y.grad).all() and (y.grad[:, 27] == 0).all()
    z = whole[:, :27].clone().requires_grad_()
    L.distill_loss(z, ids, values, lse=lse).sum().backward()
    assert ((y.grad[:, :27] - z.grad).abs() <= 1e-6).all()


def test_shards_that_can_be_gone_through_once_are_refused():
    x = torch.randn(2, 8, device="cuda")
    with pytest.raises(ValueError):
        L.process(iter([x, x]))


def test_bias_values_without_ids_are_refused():
    x = torch.randn(2, 8, device="cuda")
    with pytest.raises(ValueError, match="bias_ids"):
        L.process(x, bias_values=torch.ones(2, 3, device="cuda"))
    none = torch.empty(2, 0, device="cuda")
    assert torch.equal(L.process(x, bias_ids=none.int(), bias_values=none)[0], x)
