"""More of the steps on logits: vocabularies whose counters take several rounds, the penalties' quotients over the whole
range of fp32, what is refused on the device's side, the torch layer's refusals, and results that do not depend on the
batch.  Definitions and tolerances as in test_gpu_logits.py; what is compared here is equal bit for bit."""
import numpy as np
import pytest
import torch

import logits_util as U
from paper_2609_34645_b200 import binding as B
from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu


def _dev(a):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda")


@pytest.mark.parametrize("vocab,tp,dtype,long", [(3_000_001, 1, "bf16", False), (2_999_999, 3, "fp32", False),
                                                 (1_500_000, 2, "bf16", True)])
def test_process_in_rounds(vocab, tp, dtype, long):
    """More columns than a cluster has counters for: the history is gone through once per round."""
    rng = np.random.default_rng([7, vocab, tp])
    n = 33000 if long else 900                                   # 33000: four bytes a counter
    x = rng.normal(0, 2, (1, vocab)).astype(np.float32)
    h = rng.integers(0, vocab, (1, n)).astype(np.int32)
    h[0, : n // 3] = rng.integers(0, 50, n // 3)
    ids = rng.choice(vocab, 40, replace=False).astype(np.int32)[None]
    words = rng.integers(-2 ** 31, 2 ** 31, (1, (vocab + 31) // 32)).astype(np.int32)
    how = {"history": h, "prompt_len": np.array([n // 2], np.int32), "repetition": np.array([1.3], np.float32),
           "presence": np.array([0.4], np.float32), "frequency": np.array([0.01], np.float32), "bias_ids": ids,
           "bias_values": rng.normal(0, 3, (1, 40)).astype(np.float32), "mask": words}
    view = U.View(1, vocab, tp, dtype, "shards").put(torch.from_numpy(x))
    kept = view.get().float().cpu().numpy()
    # the definition by counting, every step rounded on its own
    want = kept[0].copy()
    seen, made = np.zeros(vocab, bool), np.bincount(h[0, n // 2:], minlength=vocab)
    seen[h[0]] = True
    want[seen] = np.where(want[seen] > 0, want[seen] / how["repetition"], want[seen] * how["repetition"])
    some = made > 0
    want[some] = (want[some] - how["frequency"] * made[some].astype(np.float32)) - how["presence"]
    want[ids[0]] = want[ids[0]] + how["bias_values"][0]
    v = np.arange(vocab)
    want[(words[0].astype(np.int64)[v >> 5] >> (v & 31) & 1) == 0] = -np.inf
    out = U.View(1, vocab, tp, dtype, "shards", fill=U.SENTINEL)
    _, token, _ = L.process(view.arg(), vocab=vocab, out=out.arg(), **{k: _dev(a) for k, a in how.items()})
    want = U.rounded(torch.from_numpy(want[None]), dtype)
    assert np.array_equal(out.get().double().cpu().numpy(), want)
    assert token.item() == want.argmax()


def test_penalties_quotients_are_rounded_as_ieee_division_rounds_them():
    """x / rho for x of any exponent, subnormal and infinite included, and rho from 2^-126 to 2^126."""
    rng = np.random.default_rng(11)
    rows, vocab = 96, 6000
    x = rng.integers(0, 1 << 32, (rows, vocab), dtype=np.uint32).view(np.float32)
    x = np.where(np.isnan(x), np.float32(1.5), x)
    x[: rows // 2] = rng.normal(0, 5, (rows // 2, vocab)).astype(np.float32)       # and the ordinary range
    rho = np.exp2(rng.uniform(-126, 126, rows)).astype(np.float32)
    rho[: rows // 2] = rng.uniform(0.5, 2, rows // 2).astype(np.float32)
    rho[0] = 1.0
    h = np.tile(np.arange(vocab, dtype=np.int32), (rows, 1))
    with np.errstate(all="ignore"):
        want = np.where(x > 0, x / rho[:, None], x * rho[:, None])
    out, _, _ = L.process(_dev(x), history=_dev(h), prompt_len=_dev(np.full(rows, vocab, np.int32)), repetition=_dev(rho))
    assert np.array_equal(out.cpu().numpy(), want)


def test_rows_beyond_shared_memory_are_refused():
    """Rows of 2^24 tokens: their records and notes, or flags, are more than a block's shared memory."""
    x = torch.zeros(1, 1 << 24, device="cuda")
    ids, values = torch.zeros(1, 3, dtype=torch.int32, device="cuda"), torch.zeros(1, 3, device="cuda")
    for call in (lambda: L.teacher_top(x, 1), lambda: L.distill_forward(x, ids, values), lambda: L.distill_step(x, ids, values)):
        with pytest.raises(B.NereusError) as e:
            call()
        assert e.value.code == B.ERR_TOO_LARGE


@pytest.mark.parametrize("tp", [1, 64])
def test_the_largest_vocabulary_that_always_fits(tp):
    vocab = 1 << 18
    rng = np.random.default_rng([13, tp])
    view = U.View(2, vocab, tp, "fp32", "odd").put(torch.from_numpy(rng.normal(0, 2, (2, vocab))))
    x = view.get()
    values, ids, lse = L.teacher_top(view.arg(), 20)
    want = x.topk(20, dim=1)
    assert torch.equal(values, want.values) and torch.equal(ids.long(), want.indices)
    loss, grad = L.distill_step(view.arg(), ids, values, lse=lse)          # its own teacher
    assert (loss.abs() < 1e-4).all()


def test_torch_layer_refusals():
    x = torch.zeros(4, 100, device="cuda")
    ids, values = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    bad = [lambda: L.process(x.half()), lambda: L.process(x[0]), lambda: L.process(x.t()), lambda: L.process([]),
           lambda: L.process([x, x[:2]]), lambda: L.process([x, x.bfloat16()]), lambda: L.process(x, out=x.cpu()),
           lambda: L.process(x, repetition=torch.ones(3, device="cuda")), lambda: L.process(x, repetition=torch.ones(4)),
           lambda: L.process(x, repetition=torch.ones(4, device="cuda", dtype=torch.float64)),
           lambda: L.process(x, history=torch.zeros(4, 2, device="cuda")), lambda: L.process(x, total_len=ids[:, 0]),
           lambda: L.process(x, mask=torch.zeros(4, 3, dtype=torch.int32, device="cuda")), lambda: L.process(x, mask_row=ids[:, 0]),
           lambda: L.process(x, bias_ids=ids), lambda: L.distill_forward(x, ids.long(), values),
           lambda: L.distill_forward(x, ids, values.t()), lambda: L.distill_forward(x, ids, values, divergence="kl"),
           lambda: L.distill_step(x, ids, values, weight=torch.ones(4))]
    for call in bad:
        with pytest.raises((ValueError, B.NereusError)):
            call()
    for k in (0, 101, -2, 10 ** 12):
        with pytest.raises(B.NereusError) as e:
            L.teacher_top(x, k)
        assert e.value.code == B.ERR_ARG
    with pytest.raises(B.NereusError) as e:
        L.distill_forward(x, ids, values, divergence="js")
    assert e.value.code == B.ERR_UNSUPPORTED
    with pytest.raises(B.NereusError) as e:
        L.process(x, vocab=101)
    assert e.value.code == B.ERR_ARG
    with pytest.raises(B.NereusError) as e:
        L.process(x[:, :50], out=x[:, 1:51])
    assert e.value.code == B.ERR_ALIAS
    torch.cuda.synchronize()


def test_a_row_gives_the_same_bits_in_any_batch():
    """Rows that start on 16-byte boundaries, in the batch and alone."""
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(300, 32008, device="cuda", generator=gen).bfloat16()
    values, ids, lse = L.teacher_top(x, 33)
    y = (x.float() + torch.randn(x.shape, device="cuda", generator=gen)).bfloat16()
    loss, grad = L.distill_step(y, ids, values, lse=lse)
    out, token, norm = L.process(x)
    for a, b in ((0, 1), (17, 40), (299, 300)):
        part = L.teacher_top(x[a:b].contiguous(), 33)
        assert all(torch.equal(p, w[a:b]) for p, w in zip(part, (values, ids, lse)))
        part = L.distill_step(y[a:b].contiguous(), ids[a:b].contiguous(), values[a:b].contiguous(), lse=lse[a:b].contiguous())
        assert torch.equal(part[0], loss[a:b]) and torch.equal(part[1], grad[a:b])
        part = L.process(x[a:b].contiguous())
        assert all(torch.equal(p, w[a:b]) for p, w in zip(part, (out, token, norm)))
