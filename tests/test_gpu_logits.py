"""The steps on an LM head's logits against their definitions in 64 bits (tests/logits_util.py).

Tolerances, derived before the first run.  EPS = 2^-24 is half a unit in the last place of fp32.
  * `process`: the definition rounds every step, so the written logits have to be equal bit for bit, and with them the
    token.  `teacher_top`: values and ids are equal.
  * sums of exponentials: relative error sum_error(V), plus the argument's rounding, 2 EPS |x - m| / T relative.
    A log-sum-exp adds the rounding of its own value.
  * distillation: with A the largest |x - m| / T, |y| / T + |lse| or |log| in play, a log-probability is off by
    e = sum_error + 8 EPS (1 + A), a probability by that times itself, P_rest = 1 - sum P by e in all.  The loss moves
    by at most (2 + A) times that, the gradient by 4 e (2 + A) of its probabilities, P_rest's error over P_rest where
    the reverse KL divides by it (the inputs keep it above 2^-9), and the written type's own rounding.
"""
import numpy as np
import pytest
import torch

import logits_util as U
from paper_2609_34645_b200 import binding as B
from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu
INF = float("inf")

# rows, vocab, tp, padded
SHAPES = [(1, 1, 1, False), (3, 7, 1, False), (2, 129, 2, True), (5, 1000, 4, False), (3, 4099, 1, False),
          (4, 50257, 4, True), (2, 32064, 8, False), (1, 128256, 1, False), (37, 8192, 1, False), (2, 300, 64, True),
          (160, 2051, 1, False), (3, 152064, 2, False)]
LAYOUTS = ["shards", "columns", "odd"]



def _seed(*key):
    import zlib
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def _logits(rng, rows, vocab, spread=2.0, peaks=3):
    x = rng.normal(0, spread, (rows, vocab))
    for r in range(rows):
        x[r, rng.integers(0, vocab, peaks)] += rng.uniform(3, 8, peaks)
    return x


def _dev(a, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda" if dtype is None else "cuda", dtype)


def _same(got, want):
    """Equal bit for bit up to the sign of zero and the payload of NaN."""
    return np.array_equal(got, want, equal_nan=True)


# ---- process ---------------------------------------------------------------------------------------------------

def _penalties(rng, rows, vocab, n, what):
    how = {}
    if "history" in what:
        h = rng.integers(0, vocab, (rows, n))
        h[rng.random((rows, n)) < 0.3] = rng.integers(0, min(vocab, 5))             # repeated often
        h[rng.random((rows, n)) < 0.05] = -1
        h[rng.random((rows, n)) < 0.05] = vocab + 3                                 # no token
        how["history"] = h.astype(np.int32)
        if "lens" in what:
            how["total_len"] = rng.integers(0, n + 1, rows).astype(np.int32)
            how["total_len"][0] = n + 7                                             # clamped
            how["prompt_len"] = rng.integers(0, n + 1, rows).astype(np.int32)
        how["repetition"] = rng.uniform(0.8, 1.5, rows).astype(np.float32)
        how["presence"] = rng.normal(0, 1, rows).astype(np.float32)
        how["frequency"] = rng.normal(0, 1, rows).astype(np.float32)
    if "bias" in what:
        k = min(vocab, 11)
        how["bias_ids"] = rng.integers(-1, vocab + 1, (rows, k)).astype(np.int32)   # some unused, some twice
        how["bias_values"] = rng.normal(0, 5, (rows, k)).astype(np.float32)
    if "mask" in what:
        g = max(1, rows - 1)
        words = rng.integers(-2 ** 31, 2 ** 31, (g, (vocab + 31) // 32 + 1)).astype(np.int32)
        words[0] = 0                                                                # leaves nothing
        how["mask"] = words
        how["mask_row"] = rng.integers(-1, g + 1, rows).astype(np.int32)
        how["mask_row"][0] = 0
    return how


def _check_process(x64, view, out_view, how, dtype, out_dtype):
    rows, vocab = x64.shape
    kept = U.rounded(x64, dtype)
    want = U.process_definition(kept.astype(np.float32), how)
    want = U.rounded(torch.from_numpy(want), out_dtype)
    out, token, lse = L.process(view.arg(), vocab=vocab, out=out_view.arg(), **{k: _dev(v) for k, v in how.items()})
    torch.cuda.synchronize()
    got = out_view.get().double().cpu().numpy()
    assert _same(got, want)
    assert out_view.untouched_outside()
    allowed = ~np.isnan(want) & (want > -INF)
    first = np.where(allowed.any(1), np.argmax(np.where(allowed, want, -INF), axis=1), -1)
    assert np.array_equal(token.cpu().numpy(), first)
    ref = U.log_sum_exp(want)
    got = lse.double().cpu().numpy()
    assert _same(np.where(np.isfinite(ref), 0, got), np.where(np.isfinite(ref), 0, ref))
    fine = np.isfinite(ref)
    spread = 20.0
    tol = U.sum_error(vocab) + 2 * U.EPS * spread + 2 * U.EPS * np.abs(ref[fine])
    assert (np.abs(got[fine] - ref[fine]) <= tol).all()


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("rows,vocab,tp,padded", SHAPES)
def test_process_over_shapes_and_layouts(rows, vocab, tp, padded, types):
    for layout in LAYOUTS:
        rng = _seed("process", rows, vocab, tp, types, layout)
        x = _logits(rng, rows, vocab)
        view = U.View(rows, vocab, tp, types[0], layout, padded).put(torch.from_numpy(x))
        out = U.View(rows, vocab, tp, types[1], layout, padded, fill=U.SENTINEL)
        how = _penalties(rng, rows, vocab, 61, ("history", "lens", "bias", "mask"))
        _check_process(x, view, out, how, *types)


@pytest.mark.parametrize("what", [(), ("history",), ("history", "lens"), ("bias",), ("mask",), ("bias", "mask")])
def test_process_with_parts_left_out(what):
    rng = _seed("parts", what)
    x = _logits(rng, 5, 1013)
    view = U.View(5, 1013, 1, "bf16", "shards").put(torch.from_numpy(x))
    out = U.View(5, 1013, 1, "fp32", "odd", fill=U.SENTINEL)                        # rows not congruent mod 16 bytes
    _check_process(x, view, out, _penalties(rng, 5, 1013, 33, what), "bf16", "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_process_in_place(dtype):
    rng = _seed("in place", dtype)
    x = _logits(rng, 9, 5003)
    view = U.View(9, 5003, 1, dtype, "odd", fill=U.SENTINEL).put(torch.from_numpy(x))
    _check_process(x, view, view, _penalties(rng, 9, 5003, 40, ("history", "lens", "bias", "mask")), dtype, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_process_with_infinities_and_nan(dtype):
    """NaN in masked places leaves no trace; NaN elsewhere reaches its row's log-sum-exp and is never the token."""
    rng = _seed("special", dtype)
    x = _logits(rng, 8, 700)
    x[0, 5] = np.nan
    x[1, 6] = INF
    x[2, 7] = -INF
    x[3, :] = -INF
    x[4, 9] = np.nan                       # masked below
    x[5, :] = np.nan
    x[6, 3:] = -INF
    x[7, :] = torch.finfo(torch.bfloat16).min
    how = {"mask": np.full((1, 22), -1, np.int32), "mask_row": np.array([-1, -1, -1, -1, 0, -1, -1, -1], np.int32)}
    how["mask"][0, 0] &= ~(1 << 9)
    view = U.View(8, 700, 1, dtype, "shards").put(torch.from_numpy(x))
    out = U.View(8, 700, 1, dtype, "shards", fill=U.SENTINEL)
    _check_process(x, view, out, how, dtype, dtype)


def test_process_long_history_counts_exactly():
    """A history longer than the block, one token far more often than 16 bits hold."""
    vocab, n = 9001, 80000
    rng = _seed("long")
    x = _logits(rng, 2, vocab)
    h = np.full((2, n), 4500, np.int32)
    h[1] = np.arange(n) % vocab
    how = {"history": h, "frequency": np.array([2.0 ** -10, 0.25], np.float32), "prompt_len": np.array([5, 77], np.int32)}
    kept = U.rounded(x, "fp32").astype(np.float32)
    want = kept.copy()
    for r in range(2):
        count = np.bincount(h[r, how["prompt_len"][r]:], minlength=vocab).astype(np.float32)
        want[r] = kept[r] - how["frequency"][r] * count
    out, token, _ = L.process(_dev(kept), **{k: _dev(v) for k, v in how.items()})
    assert np.array_equal(out.cpu().numpy(), want)
    assert np.array_equal(token.cpu().numpy(), want.argmax(1))


def test_process_bias_list_at_its_limit():
    vocab, n = 2000, B.BIAS_MAX
    rng = _seed("bias limit")
    x = _logits(rng, 2, vocab)
    ids = np.stack([rng.permutation(vocab)[:n], np.full(n, 17)]).astype(np.int32)   # all distinct; all one token
    how = {"bias_ids": ids, "bias_values": rng.normal(0, 3, (2, n)).astype(np.float32),
           "history": ids[:, :50].copy(), "repetition": np.array([1.3, 1.1], np.float32)}
    view = U.View(2, vocab, 1, "fp32", "shards").put(torch.from_numpy(x))
    out = U.View(2, vocab, 1, "fp32", "shards", fill=U.SENTINEL)
    _check_process(x, view, out, how, "fp32", "fp32")


def test_process_ties_go_to_the_lowest_id():
    x = torch.zeros(4, 40000, device="cuda")
    x[0, 39999] = x[0, 20001] = 1.0
    x[1, 0] = x[1, 39999] = 2.0
    x[2, 777] = -1.0
    x[3] = -0.0
    x[3, 100] = 0.0
    _, token, _ = L.process(x)
    assert token.tolist() == [20001, 0, 0, 0]


# ---- teacher_top -----------------------------------------------------------------------------------------------

def _top_definition(x, k):
    """Largest first, equal ones by rising id, NaN never."""
    rows, vocab = x.shape
    values, ids = np.full((rows, k), -INF), np.full((rows, k), -1)
    for r in range(rows):
        ok = np.flatnonzero(~np.isnan(x[r]))
        order = ok[np.argsort(-(x[r][ok] + 0.0), kind="stable")][:k]
        values[r, :len(order)], ids[r, :len(order)] = x[r][order], order
    return values, ids


def _check_top(x64, view, k, dtype, temperature=1.0):
    rows, vocab = x64.shape
    kept = U.rounded(x64, dtype)
    values, ids, lse = L.teacher_top(view.arg(), k, vocab=vocab, temperature=temperature)
    want_v, want_i = _top_definition(kept, k)
    assert np.array_equal(ids.cpu().numpy(), want_i)
    assert np.array_equal(values.double().cpu().numpy(), want_v)
    ref = U.log_sum_exp(kept / np.float64(np.float32(temperature)))
    got = lse.double().cpu().numpy()
    fine = np.isfinite(ref)
    assert _same(got[~fine], ref[~fine])
    spread = 30.0 / temperature
    tol = U.sum_error(vocab) + 4 * U.EPS * spread + 4 * U.EPS * np.abs(ref[fine])
    assert (np.abs(got[fine] - ref[fine]) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,tp,padded", SHAPES)
def test_top_over_shapes_and_layouts(rows, vocab, tp, padded, dtype):
    for layout in LAYOUTS:
        rng = _seed("top", rows, vocab, tp, dtype, layout)
        x = _logits(rng, rows, vocab)
        view = U.View(rows, vocab, tp, dtype, layout, padded).put(torch.from_numpy(x))
        for k in {1, min(vocab, 20), min(vocab, 64), min(vocab, B.TOP_MAX_K)}:
            _check_top(x, view, k, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["constant", "two", "rising", "falling", "block", "few", "steps", "clustered"])
@pytest.mark.parametrize("vocab,tp", [(2049, 1), (50000, 2), (128256, 4)])
def test_top_of_rows_that_are_hard_to_cut(kind, vocab, tp, dtype):
    """Rows with far more equal values than k, in order, or with their largest values side by side."""
    rng = _seed("hard", kind, vocab, dtype)
    v = np.arange(vocab)
    x = {"constant": np.full(vocab, 1.5), "two": (v % 2).astype(float), "rising": v / vocab * 8, "falling": -v / vocab * 8,
         "block": np.where((v > 100) & (v < 700), 9.0 + (v % 5), rng.normal(0, 1, vocab)),
         "few": np.where(v % (vocab // 3) == 5, 3.0, -INF), "steps": np.round(rng.normal(0, 1, vocab)),
         "clustered": np.where(v >= vocab - 300, 20 - (v % 7) * 0.25, 0.0)}[kind]
    x = np.stack([x, x[::-1], np.roll(x, 1)])
    view = U.View(3, vocab, tp, dtype, "shards").put(torch.from_numpy(x))
    for k in (1, 63, 200):
        _check_top(x, view, k, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_top_with_infinities_nan_and_signed_zeros(dtype):
    rng = _seed("top special", dtype)
    x = rng.normal(0, 1, (7, 600))
    x[0, 3] = np.nan
    x[1, :] = np.nan
    x[2, 10:] = np.nan
    x[3, 5], x[3, 50] = INF, INF
    x[4, :] = -INF
    x[5, :] = np.where(np.arange(600) % 2, 0.0, -0.0)
    x[6, 4:] = -INF
    view = U.View(7, 600, 1, dtype, "odd").put(torch.from_numpy(x))
    for k in (1, 16, 256):
        _check_top(x, view, k, dtype)


@pytest.mark.parametrize("temperature", [0.25, 0.7, 3.0])
def test_top_temperature(temperature):
    rng = _seed("temperature", temperature)
    x = _logits(rng, 4, 3001)
    _check_top(x, U.View(4, 3001, 1, "fp32", "shards").put(torch.from_numpy(x)), 10, "fp32", temperature)


# ---- distillation ----------------------------------------------------------------------------------------------

HOW = [("forward_kl", True, 1.0, 0.5), ("forward_kl", False, 2.0, 0.5), ("reverse_kl", True, 1.0, 0.5),
       ("js", True, 0.7, 0.3)]


def _teacher(rng, x, k, temperature):
    """Entries of a teacher near the student: values, ids, log-sum-exp."""
    y = (x + rng.normal(0, 1, x.shape)).astype(np.float32).astype(np.float64)
    ids = np.argsort(-y, axis=1, kind="stable")[:, :k]
    lse = U.log_sum_exp(y / temperature).astype(np.float32)
    return np.take_along_axis(y, ids, 1).astype(np.float32), ids.astype(np.int32), lse


def _bounds(kept, ids, values, lse, temperature, vocab):
    a = np.abs(kept - kept.max(1, keepdims=True)).max() / temperature + np.abs(values).max() / temperature
    a += np.abs(lse).max() + 17.0
    e = U.sum_error(vocab) + 8 * U.EPS * (1 + a)
    return a, e


def _check_distill(x64, make, ids, values, lse, weight, divergence, temperature, beta, dtype, in_place=False):
    rows, vocab = x64.shape
    kept = U.rounded(x64, dtype)
    t = float(np.float32(temperature))
    d, g, sums = U.distill_definition(kept, ids, values.astype(np.float64), None if lse is None else lse.astype(np.float64),
                                      t, divergence, float(np.float32(beta)))
    w = np.ones(rows) if weight is None else weight.astype(np.float64)
    live = w != 0
    a, e = _bounds(kept[live], ids, values, np.zeros(1) if lse is None else lse, temperature, vocab) if live.any() else (0, 0)
    how = {"vocab": vocab, "lse": None if lse is None else _dev(lse), "weight": None if weight is None else _dev(weight),
           "divergence": divergence, "temperature": temperature, "beta": beta}
    di, dv = _dev(ids), _dev(values)
    last = 2.0 ** -9 if dtype == "bf16" else 2 * U.EPS
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149

    def check_loss(loss):
        got = loss.double().cpu().numpy()
        assert (got[~live] == 0).all()
        assert (np.abs(got - d * w)[live] <= (np.abs(w) * ((2 + a) * 2 * e + 4 * U.EPS * np.abs(d)))[live]).all()

    def check_grad(view, scale):
        got = view.get().double().cpu().numpy()
        assert (got[~live] == 0).all()
        want = g * scale[:, None]
        q = np.exp((kept - kept.max(1, keepdims=True)) / t)
        q = q / q.sum(1, keepdims=True)
        p = np.zeros_like(q)
        for r in range(rows):
            use = (ids[r] >= 0) & (ids[r] < vocab)
            p[r, ids[r][use]] = 1.0 if lse is None else np.exp(np.minimum(0, values[r][use] / t - lse[r]))
        tol = (4 * e * (2 + a) * (q + p) + q * e * 2.0 ** 9) * np.abs(scale)[:, None] / t + last * np.abs(want) + tiny
        assert (np.abs(got - want)[live] <= tol[live]).all()
        assert view.untouched_outside()

    src = make(float("nan")).put(torch.from_numpy(np.where(live[:, None], x64, np.nan)))
    loss, saved = L.distill_forward(src.arg(), di, dv, **how)
    check_loss(loss)
    got = saved.double().cpu().numpy()
    assert (got[~live] == 0).all()
    assert np.array_equal(got[live, 0], sums[live, 0])
    assert (np.abs(got - sums)[live, 1:3] <= (e * sums[live, 1:3] + 2.0 ** -149)).all()

    up = _seed("up", rows).uniform(-2, 2, rows).astype(np.float32)
    out = make(U.SENTINEL)
    L.distill_backward(src.arg(), di, dv, saved, grad_loss=_dev(up), grad=out.arg(), **how)
    check_grad(out, w * up)
    out = make(U.SENTINEL)
    if in_place:
        out.put(torch.from_numpy(x64))
        loss, _ = L.distill_step(out.arg(), di, dv, grad=out.arg(), **how)
    else:
        loss, _ = L.distill_step(src.arg(), di, dv, grad=out.arg(), **how)
    check_loss(loss)
    check_grad(out, w)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,tp,padded", [s for s in SHAPES if s[1] > 1])
def test_distill_over_shapes_and_layouts(rows, vocab, tp, padded, dtype):
    for n, (divergence, rest, temperature, beta) in enumerate(HOW):
        layout = LAYOUTS[(n + rows) % 3]
        rng = _seed("distill", rows, vocab, tp, dtype, n)
        x = _logits(rng, rows, vocab)
        k = min(vocab // 2, (1, 5, 33, 256)[(n + vocab) % 4])
        values, ids, lse = _teacher(rng, U.rounded(x, dtype), k, temperature)
        weight = rng.uniform(-0.5, 2, rows).astype(np.float32)
        weight[1::3] = 0
        _check_distill(x, lambda fill: U.View(rows, vocab, tp, dtype, layout, padded, fill), ids, values,
                       lse if rest else None, weight, divergence, temperature, beta, dtype, in_place=n % 2 == 1)


@pytest.mark.parametrize("divergence,rest,temperature,beta", HOW)
def test_distill_entries_left_out_and_every_token_an_entry(divergence, rest, temperature, beta):
    rng = _seed("entries", divergence, rest)
    rows, vocab, k = 6, 40, 40
    x = _logits(rng, rows, vocab)
    values, ids, lse = _teacher(rng, x, k, temperature)
    ids[1, 3:] = -1                         # three entries
    ids[2, :] = -1                          # none
    ids[3, ::2] = vocab + 2                 # every other one
    ids[4, 7] = -5
    _check_distill(x, lambda fill: U.View(rows, vocab, 1, "fp32", "shards", False, fill), ids, values,
                   lse if rest else None, None, divergence, temperature, beta, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_distill_masked_student_logits(dtype):
    """-inf logits of tokens the teacher does not name cost nothing; of one that it names, an infinite forward KL and a
    gradient that is still finite."""
    rng = _seed("masked", dtype)
    x = _logits(rng, 4, 500)
    values, ids, lse = _teacher(rng, U.rounded(x, dtype), 8, 1.0)
    x[0, [v for v in range(100) if v not in ids[0]]] = -INF
    x[1, [v for v in range(500) if v not in ids[1]]] = -INF       # nothing left to the rest
    x[2, ids[2, 3]] = -INF
    dev = _dev(x.astype(np.float32)).to(U.TYPES[dtype])
    for divergence in ("forward_kl", "js", "reverse_kl"):
        d, g, _ = U.distill_definition(U.rounded(x, dtype), ids, values.astype(np.float64), lse.astype(np.float64), 1.0,
                                       divergence, 0.5)
        loss, grad = L.distill_step(dev, _dev(ids), _dev(values), lse=_dev(lse), divergence=divergence)
        got, grad = loss.double().cpu().numpy(), grad.double().cpu().numpy()
        assert np.array_equal(np.isinf(got), np.isinf(d))
        fine = np.isfinite(d)
        assert np.allclose(got[fine], d[fine], rtol=1e-4, atol=1e-5)
        if divergence == "forward_kl":
            assert np.isfinite(grad).all()
            assert np.isinf(d[1]) and np.isinf(d[2])
            g[1, [v for v in range(500) if v not in ids[1]]] = 0.0     # tokens without mass have no gradient
            assert np.allclose(grad, g, rtol=2.0 ** -7, atol=1e-4)
        else:
            assert np.allclose(grad[fine], g[fine], rtol=2.0 ** -7, atol=1e-4)


def test_distill_rows_of_weight_zero_are_not_read():
    x = torch.full((3, 1000), float("nan"), device="cuda")
    ids = torch.randint(1000, (3, 4), device="cuda", dtype=torch.int32)
    values, lse = torch.full((3, 4), float("nan"), device="cuda"), torch.full((3,), float("inf"), device="cuda")
    loss, grad = L.distill_step(x, ids, values, lse=lse, weight=torch.zeros(3, device="cuda"))
    assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize("divergence,rest,temperature,beta", HOW)
def test_distill_gradient_against_differences(divergence, rest, temperature, beta):
    """Central differences of the 64-bit loss; their own error is h^2 / 6 times the third derivative (of order 1 / T^3)
    plus the loss's rounding over h."""
    rng = _seed("differences", divergence)
    rows, vocab, k, h = 2, 60, 6, 1e-4
    x = _logits(rng, rows, vocab).astype(np.float32).astype(np.float64)
    values, ids, lse = _teacher(rng, x, k, temperature)
    args = (ids, values.astype(np.float64), lse.astype(np.float64) if rest else None, temperature, divergence, beta)
    _, grad = L.distill_step(_dev(x.astype(np.float32)), _dev(ids), _dev(values), lse=_dev(lse) if rest else None,
                             divergence=divergence, temperature=temperature, beta=beta)
    grad = grad.double().cpu().numpy()
    for v in range(vocab):
        up, down = x.copy(), x.copy()
        up[:, v] += h
        down[:, v] -= h
        diff = (U.distill_definition(up, *args)[0] - U.distill_definition(down, *args)[0]) / (2 * h)
        assert (np.abs(diff - grad[:, v]) < 1e-5).all()


def test_distill_loss_under_autograd():
    """Through a product with the head, over two shards of a padded vocabulary: the gradient of the hidden states and
    of both shards of the head."""
    rng = _seed("autograd")
    rows, hidden, vocab = 6, 16, 200
    w = U.width(vocab, 2, True)
    h = torch.randn(rows, hidden, device="cuda", dtype=torch.float32, requires_grad=True)
    head = [torch.randn(w, hidden, device="cuda", requires_grad=True) for _ in range(2)]
    values, ids, lse = _teacher(rng, (h @ torch.cat(head).T)[:, :vocab].detach().cpu().double().numpy(), 5, 1.0)
    values, ids, lse = _dev(values), _dev(ids), _dev(lse)
    weight = torch.tensor([1.0, 0.0, 2.0, 0.5, 1.0, 1.0], device="cuda")
    shards = [h @ p.T for p in head]
    L.distill_loss(shards, ids, values, vocab=vocab, lse=lse, weight=weight).sum().backward()
    got = [h.grad, head[0].grad, head[1].grad]

    h2, p2 = h.detach().double().requires_grad_(), [p.detach().double().requires_grad_() for p in head]
    logq = torch.log_softmax(torch.cat([h2 @ p.T for p in p2], 1)[:, :vocab], 1)
    top = logq.gather(1, ids.long())
    rest = torch.logsumexp(logq.scatter(1, ids.long(), -INF), 1, keepdim=True)
    p = torch.exp(values.double() - lse.double()[:, None])
    p = torch.cat([p, (1 - p.sum(1, keepdim=True)).clamp(min=0)], 1)
    loss = torch.special.xlogy(p, p).sum(1) - (p * torch.cat([top, rest], 1)).sum(1)
    (loss * weight).sum().backward()
    for a, b in zip(got, [h2.grad, p2[0].grad, p2[1].grad]):
        assert torch.isfinite(a).all()
        assert (a.double() - b).abs().max() <= 1e-4 * b.abs().max()
    assert (got[2][vocab - w:] == 0).all()                    # padding rows of the head take no part


# ---- streams, graphs, repetition -------------------------------------------------------------------------------

def test_same_results_on_another_stream_and_from_a_captured_graph():
    rng = _seed("graph")
    x = _dev(_logits(rng, 33, 9001).astype(np.float32)).bfloat16()
    values, ids, lse = L.teacher_top(x, 17)
    x2 = (x.float() + 0.5 * torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1))).bfloat16()
    loss, grad = L.distill_step(x2, ids, values, lse=lse)
    out, token, norm = L.process(x)
    torch.cuda.synchronize()

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = L.teacher_top(x, 17)
        b = L.distill_step(x2, a[1], a[0], lse=a[2])
        c = L.process(x)
    side.synchronize()
    for got, want in zip((*a, *b, *c), (values, ids, lse, loss, grad, out, token, norm)):
        assert torch.equal(got, want)

    graph = torch.cuda.CUDAGraph()
    keep = x.clone(), x2.clone()
    with torch.cuda.graph(graph):
        a = L.teacher_top(x, 17)
        b = L.distill_step(x2, a[1], a[0], lse=a[2])
        c = L.process(x)
    x.zero_()
    x2.zero_()
    graph.replay()
    assert (a[0] == 0).all() and (b[0].abs() < 1e-6).all() and (c[1] == 0).all()
    x.copy_(keep[0])
    x2.copy_(keep[1])
    graph.replay()
    torch.cuda.synchronize()
    for got, want in zip((*a, *b, *c), (values, ids, lse, loss, grad, out, token, norm)):
        assert torch.equal(got, want)


def test_offsets_beyond_32_bits():
    """A bf16 tensor of more than 2^32 bytes (and 2^31 elements): its last rows give what they give alone."""
    rows, vocab = 17500, 128256
    x = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator("cuda").manual_seed(3)
    tail = torch.randn(5, vocab, device="cuda", generator=gen).bfloat16()
    x.zero_()
    x[-5:] = tail
    values, ids, lse = L.teacher_top(x, 9)
    one = L.teacher_top(tail, 9)
    for got, want in zip((values, ids, lse), one):
        assert torch.equal(got[-5:], want)
    out, token, norm = L.process(x, out=x)
    two = L.process(tail)
    assert torch.equal(out[-5:], two[0]) and torch.equal(token[-5:], two[1]) and torch.equal(norm[-5:], two[2])
    weight = torch.zeros(rows, device="cuda")
    weight[-5:] = 1
    loss, grad = L.distill_step(x, ids, values, lse=lse, weight=weight, grad=x)
    three = L.distill_step(tail, one[1], one[0], lse=one[2])
    assert torch.equal(loss[-5:], three[0]) and torch.equal(grad[-5:], three[1])
    assert (grad[:64] == 0).all()
