"""A row gives the same bits alone and in any batch in which its shards start alike modulo 16 bytes: with rows of an odd
stride among them, at widths that fill layers exactly.  No tolerance."""
import pytest
import torch

from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu


def _cut(whole, w):
    return list(whole.split(w, dim=1))


# a layer holds 4096 bf16 or 2048 fp32 (8192 and 4096 in the distillation's backward pass and step)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab,tp", [(4096, 1), (8192, 1), (16384, 1), (32768, 1), (65536, 1), (131072, 1), (131072, 2), (32768, 8),
                                      (16384, 4), (16400, 1), (50264, 1)])
def test_rows_with_an_odd_stride(vocab, tp, dtype):
    rows, w, step = 17, vocab // tp, 8                      # a row of an odd stride starts on 16 bytes every eight rows
    gen = torch.Generator("cuda").manual_seed(vocab + tp)
    # the batch: each shard a slice of rows vocab / tp + 1 long
    batch = [torch.empty(rows, w + 1, device="cuda", dtype=dtype)[:, :w].copy_(torch.randn(rows, w, device="cuda", generator=gen) * 3)
             for _ in range(tp)]
    ids = torch.stack([torch.randperm(vocab, device="cuda", generator=gen)[:9] for _ in range(rows)]).int()
    values = torch.randn(rows, 9, device="cuda", generator=gen).sort(descending=True).values
    lse = torch.full((rows,), 8.0, device="cuda")
    h = torch.randint(vocab, (rows, 50), device="cuda", generator=gen, dtype=torch.int32)
    half = torch.full((rows,), 0.5, device="cuda")

    def everything(x, r):
        up = lambda t: t[r].contiguous()                                                                    # noqa: E731
        out, token, norm = L.process(x)
        out2, token2, norm2 = L.process(x, history=up(h), repetition=up(half), presence=up(half))
        top = L.teacher_top(x, 7)
        loss, saved = L.distill_forward(x, up(ids), up(values), lse=up(lse), divergence="js")
        back = L.distill_backward(x, up(ids), up(values), saved, lse=up(lse), divergence="js")
        loss2, grad = L.distill_step(x, up(ids), up(values), lse=up(lse))
        return [*out, token, norm, *out2, token2, norm2, *top, loss, saved, *back, loss2, *grad]

    want = everything(batch, slice(None))
    for r in (0, step, 2 * step):
        alone = [s[r:r + 1].contiguous() for s in batch]
        for got, all_rows in zip(everything(alone, slice(r, r + 1)), want):
            assert torch.equal(got, all_rows[r:r + 1])


@pytest.mark.parametrize("vocab,tp", [(8192, 2), (16384, 1), (16384, 4), (32768, 8)])
def test_lowest_token_and_counts_in_rows_that_start_anywhere(vocab, tp):
    """Equal largest values at both ends of every shard, and a history there, at every alignment of the row."""
    rows, w = 16, vocab // tp
    whole = torch.full((tp, rows * (w + 1) + 8), float("nan"), device="cuda", dtype=torch.bfloat16)
    x = [whole[s][1:1 + rows * (w + 1)].view(rows, w + 1)[:, :w] for s in range(tp)]
    for r in range(rows):
        for s in range(tp):
            x[s][r] = -1.0
        for s in range(r % tp, tp):
            x[s][r, -1] = 2.0
            if s > r % tp:
                x[s][r, 0] = 2.0
    first = [(r % tp) * w + w - 1 for r in range(rows)]
    _, token, _ = L.process(x)
    assert token.tolist() == first
    assert L.teacher_top(x, 1)[1][:, 0].tolist() == first
    h = torch.tensor([[t, t, 0] for t in first], device="cuda", dtype=torch.int32)
    out, token, _ = L.process(x, history=h, frequency=torch.full((rows,), 0.25, device="cuda"))
    out = torch.cat(out, 1).float()
    assert out.gather(1, h.long()).tolist() == [[1.5, 1.5, -1.25 if t else 1.5]  for t in first]
    nxt = [min((s * w for s in range(r % tp + 1, tp)), default=t) for r, t in enumerate(first)]
    assert token.tolist() == nxt
    loss, grad = L.distill_step(x, torch.tensor([[t] for t in first], device="cuda", dtype=torch.int32),
                                torch.full((rows, 1), 2.0, device="cuda"), lse=torch.full((rows,), 3.0, device="cuda"))
    g = torch.cat(grad, 1).double().sum(1).abs()
    assert (g <= 2.0 ** -8).all()
