"""What autograd has to notice: tensors that a loss has saved and that change before its backward pass, and inputs that a loss
has no gradient for."""
import pytest
import torch

from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu


def _case(shards=1):
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(5, 64, device="cuda", generator=gen, requires_grad=True)
    values, ids, lse = L.teacher_top(x.detach() + 0.3, 4)
    weight = torch.rand(5, device="cuda", generator=gen) + 0.5
    y = [s * 1.0 for s in x.split(64 // shards, dim=1)] if shards > 1 else x * 1.0
    return x, y, values, ids, lse, weight


@pytest.mark.parametrize("shards", [1, 2])
@pytest.mark.parametrize("call", ["process", "step", "backward"])
def test_logits_written_in_place_after_the_loss(call, shards):
    x, y, values, ids, lse, weight = _case(shards)
    loss = L.distill_loss(y, ids, values, lse=lse, weight=weight)
    if call == "process":
        L.process(y, out=y)
    elif call == "step":
        L.distill_step(y, ids, values, lse=lse, grad=y)
    else:
        _, saved = L.distill_forward(y, ids, values, lse=lse)
        L.distill_backward(y, ids, values, saved, lse=lse, grad=y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


@pytest.mark.parametrize("which", ["lse", "weight", "values", "ids"])
def test_a_teacher_that_changes_between_the_passes(which):
    x, y, values, ids, lse, weight = _case()
    loss = L.distill_loss(y, ids, values, lse=lse, weight=weight)
    {"lse": lse, "weight": weight, "values": values, "ids": ids}[which].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


def test_no_gradient_is_dropped_in_silence():
    x, y, values, ids, lse, weight = _case()
    for name, t in (("lse", lse), ("weight", weight), ("values", values)):
        how = {"lse": lse, "weight": weight, "values": values} | {name: t.clone().requires_grad_()}
        with pytest.raises(ValueError, match=name):
            L.distill_loss(y, ids, how.pop("values"), **how)
        with torch.no_grad():
            L.distill_loss(y, ids, **({"values": values, "lse": lse, "weight": weight} | {name: t.clone().requires_grad_()}))


def test_writing_leaves_the_rest_of_the_graph_usable():
    """Logits of a product may be overwritten by their own gradient: the product saved its factors, not its result."""
    h, w = torch.randn(5, 8, device="cuda", requires_grad=True), torch.randn(64, 8, device="cuda")
    logits = h @ w.T
    values, ids, lse = L.teacher_top(torch.randn(5, 64, device="cuda"), 4)
    _, want = L.distill_step(logits, ids, values, lse=lse)
    _, grad = L.distill_step(logits, ids, values, lse=lse, grad=logits)
    assert grad is logits and torch.equal(grad, want)
    logits.backward(gradient=grad.detach().clone())
    assert torch.equal(h.grad, want @ w)
    with torch.inference_mode():
        z = torch.randn(3, 64, device="cuda")
        assert L.process(z, out=z)[0] is z
