"""What the steps on logits refuse, and the host-side checks behind it.  No GPU: every call here is refused, or has no
rows, before anything is enqueued, so the device addresses are made up."""
import ctypes

import pytest
import torch

from paper_2609_34645_b200 import binding as B
from paper_2609_34645_b200 import logits as L

A = 1 << 30               # a made-up device address, well aligned


def view(dtype=B.BF16, tp=2, rows=4, vocab=100, cols=50, stride=None, base=A, step=1 << 20):
    v = B.Logits(dtype, tp, rows, vocab, cols, cols if stride is None else stride)
    for s in range(min(tp, B.VOCAB_MAX_TP)):
        v.shard[s] = base + s * step
    return v


def other(**kw):
    return view(base=A << 1, **kw)


def code(f, *args):
    try:
        f(*args)
    except B.NereusError as e:
        return e.code
    return B.OK


def process(src, out, how=None, token=0, lse=0):
    return code(B.logits_process, src, out, how or B.Penalties(), token, lse)


def top(src, k=4, temperature=1.0, values=A, ids=A, lse=A):
    return code(B.teacher_top, src, k, temperature, values, ids, lse)


def distill(k=4, divergence=B.FORWARD_KL, beta=0.5, temperature=1.0, values=A, ids=A, lse=A, weight=None):
    return B.Distill(k, divergence, beta, temperature, values, ids, lse, weight)


BAD_VIEWS = [
    (dict(dtype=3), B.ERR_UNSUPPORTED),
    (dict(dtype=0), B.ERR_UNSUPPORTED),
    (dict(tp=0), B.ERR_ARG),
    (dict(tp=B.VOCAB_MAX_TP + 1), B.ERR_ARG),
    (dict(rows=-1), B.ERR_ARG),
    (dict(vocab=0), B.ERR_ARG),
    (dict(cols=0), B.ERR_ARG),
    (dict(cols=49), B.ERR_ARG),                            # two shards of 49 do not hold 100 columns
    (dict(stride=49), B.ERR_ARG),                          # rows would overlap
    (dict(stride=0), B.ERR_ARG),
    (dict(stride=-50), B.ERR_ARG),
    (dict(base=A + 1), B.ERR_ALIGN),
    (dict(dtype=B.FP32, base=A + 2), B.ERR_ALIGN),
    (dict(rows=1 << 40), B.ERR_TOO_LARGE),
    (dict(vocab=1 << 30, cols=1 << 30), B.ERR_TOO_LARGE),
]


@pytest.mark.parametrize("bad, want", BAD_VIEWS)
def test_bad_views_are_refused_by_every_call(bad, want):
    src, out = view(**bad), other(**{k: v for k, v in bad.items() if k != "base"})
    assert process(src, out) == want
    assert top(src) == want
    assert code(B.distill_forward, src, distill(), A, A) == want
    assert code(B.distill_backward, src, distill(), A, A, out) == want
    assert code(B.distill_step, src, distill(), A, out) == want


def test_null_arguments():
    lib, v, w, s = B._lib, view(), other(), None
    null = view()
    null.shard[1] = None
    assert process(null, w) == process(v, null) == B.ERR_ARG
    assert lib.nereus_logits_process(None, w, B.Penalties(), s, s, s) == B.ERR_ARG
    assert lib.nereus_logits_process(v, None, B.Penalties(), s, s, s) == B.ERR_ARG
    assert lib.nereus_logits_process(v, w, None, s, s, s) == B.ERR_ARG
    assert lib.nereus_teacher_top(None, 1, 1.0, A, A, A, s) == B.ERR_ARG
    for bad in (dict(values=None), dict(ids=None), dict(lse=None)):
        assert top(v, **bad) == B.ERR_ARG
    assert lib.nereus_distill_forward(v, None, A, A, s) == B.ERR_ARG
    assert lib.nereus_distill_forward(None, distill(), A, A, s) == B.ERR_ARG
    for bad in (dict(values=None), dict(ids=None)):
        assert code(B.distill_forward, v, distill(**bad), A, A) == B.ERR_ARG
    assert code(B.distill_forward, v, distill(), None, A) == B.ERR_ARG
    assert code(B.distill_forward, v, distill(), A, None) == B.ERR_ARG
    assert code(B.distill_backward, v, distill(), None, None, w) == B.ERR_ARG
    assert lib.nereus_distill_backward(v, distill(), A, s, None, s) == B.ERR_ARG
    assert code(B.distill_step, v, distill(), None, w) == B.ERR_ARG


def test_a_padding_shard_may_be_null_but_a_used_one_may_not():
    v, w = view(tp=3), other(tp=3)
    v.shard[2] = w.shard[2] = None                          # 2 * 50 columns hold the vocabulary
    assert top(v, k=0) == B.ERR_ARG and top(v, k=101) == B.ERR_ARG
    v.rows = w.rows = 0
    assert process(v, w) == top(v) == B.OK


def test_views_that_do_not_match():
    v = view()
    for kw in (dict(rows=3), dict(vocab=99), dict(tp=4, cols=25), dict(cols=60)):
        assert process(v, other(**kw)) == B.ERR_MISMATCH
        assert code(B.distill_step, v, distill(), A, other(**kw)) == B.ERR_MISMATCH
    assert process(view(dtype=B.FP32), other(dtype=B.BF16)) == B.ERR_UNSUPPORTED
    assert code(B.distill_step, v, distill(), A, other(dtype=B.FP32)) == B.ERR_UNSUPPORTED
    assert code(B.distill_backward, view(dtype=B.FP32), distill(), A, None, other()) == B.ERR_UNSUPPORTED


def test_overlapping_views():
    v = view()
    moved = view(base=A + 2)                                # the same buffers, one element on
    assert process(v, moved) == B.ERR_ALIAS
    wide = view(stride=64)                                  # the same start, another stride
    assert process(v, wide) == B.ERR_ALIAS
    crossed = view(base=A + (1 << 20), step=-(1 << 20))     # shard 0 written over shard 1
    assert process(v, crossed) == B.ERR_ALIAS
    assert process(v, other(step=0)) == B.ERR_ALIAS         # both shards written to one place
    f = view(dtype=B.FP32)
    assert process(v, f) == B.ERR_ALIAS                     # wider elements over the ones still to be read
    slices = view(stride=99, step=100)                      # column slices of one tensor that overlap by a column
    assert process(v, other(stride=99, step=100)) == B.ERR_ALIAS
    assert process(slices, slices) == B.ERR_ALIAS


def test_column_slices_and_in_place_are_not_overlaps():
    """These pass every check; a mask that is too short is looked at after them, so its code shows how far they came."""
    short = B.Penalties()
    short.mask, short.mask_stride, short.mask_rows = A, 3, 4
    for src, out in ((view(), view()),                                              # in place
                     (view(stride=100, step=100), view(stride=100, step=100)),      # ... column slices
                     (view(stride=100, step=100), other(stride=100, step=100)),
                     (view(stride=200, step=100), view(stride=200, step=100, base=A + 200)),   # beside each other
                     (view(rows=1, stride=0), view(rows=1, stride=77))):
        assert process(src, out, short) == B.ERR_ARG
        short.mask_stride = 4
        short.bias_count = B.BIAS_MAX + 1
        short.bias_ids = short.bias_values = A
        assert process(src, out, short) == B.ERR_TOO_LARGE
        short.mask_stride, short.bias_count, short.bias_ids, short.bias_values = 3, 0, None, None


def test_penalties_arguments():
    def how(**kw):
        h = B.Penalties()
        for k, x in kw.items():
            setattr(h, k, x)
        return process(view(), other(), h)

    assert how(history=A, history_len=5, history_stride=4) == B.ERR_ARG
    assert how(history=A, history_len=-1, history_stride=4) == B.ERR_ARG
    assert how(history=A, history_len=B.HISTORY_MAX + 1, history_stride=B.HISTORY_MAX + 1) == B.ERR_TOO_LARGE
    assert how(prompt_len=A) == B.ERR_ARG
    assert how(total_len=A) == B.ERR_ARG
    assert how(bias_ids=A, bias_count=1) == B.ERR_ARG
    assert how(bias_values=A, bias_count=1) == B.ERR_ARG
    assert how(bias_ids=A, bias_values=A, bias_count=-1) == B.ERR_ARG
    assert how(bias_ids=A, bias_values=A, bias_count=B.BIAS_MAX + 1) == B.ERR_TOO_LARGE
    assert how(mask=A, mask_stride=3, mask_rows=4) == B.ERR_ARG        # 3 words hold 96 of 100 tokens
    assert how(mask=A, mask_stride=4, mask_rows=3) == B.ERR_ARG        # rows without a mask, and no mask_row
    assert how(mask=A, mask_stride=4, mask_rows=-1, mask_row=A) == B.ERR_ARG
    assert how(mask_row=A) == B.ERR_ARG
    for name in ("repetition", "presence", "frequency"):
        assert how(**{name: A + 2}) == B.ERR_ALIGN
    assert how(history=A + 1, history_len=1, history_stride=1) == B.ERR_ALIGN
    assert how(mask=A + 2, mask_stride=4, mask_rows=4) == B.ERR_ALIGN
    assert process(view(), other(), None, token=A + 1) == process(view(), other(), None, lse=A + 2) == B.ERR_ALIGN


def test_top_arguments():
    for k in (0, -1, 101, B.TOP_MAX_K + 1):
        assert top(view(), k=k) == B.ERR_ARG
    assert top(view(vocab=1000, cols=500), k=B.TOP_MAX_K + 1) == B.ERR_ARG
    for t in (0.0, -1.0, float("inf"), float("nan")):
        assert top(view(), temperature=t) == B.ERR_ARG
    assert top(view(), ids=A + 2) == B.ERR_ALIGN


def test_distill_arguments():
    def forward(**kw):
        return code(B.distill_forward, view(), distill(**kw), A, A)

    for k in (0, -3, B.TOP_MAX_K + 1):
        assert forward(k=k) == B.ERR_ARG
    for t in (0.0, -1.0, float("inf"), float("nan")):
        assert forward(temperature=t) == B.ERR_ARG
    for d in (-1, 3):
        assert forward(divergence=d) == B.ERR_ARG
    for beta in (0.0, 1.0, -0.5, float("nan")):
        assert forward(divergence=B.JENSEN, beta=beta) == B.ERR_ARG
    assert forward(divergence=B.REVERSE_KL, lse=None) == B.ERR_UNSUPPORTED
    assert forward(divergence=B.JENSEN, lse=None) == B.ERR_UNSUPPORTED
    assert forward(values=A + 2) == forward(weight=A + 1) == B.ERR_ALIGN
    assert code(B.distill_forward, view(), distill(), A + 1, A) == B.ERR_ALIGN


def test_no_rows_is_a_call_that_does_nothing():
    v, w = view(rows=0), other(rows=0)
    assert process(v, w) == top(v) == B.OK
    assert code(B.distill_forward, v, distill(), A, A) == B.OK
    assert code(B.distill_backward, v, distill(), A, None, w) == B.OK
    assert code(B.distill_step, v, distill(), A, w) == B.OK


def test_structs_have_the_header_s_layout(tmp_path):
    """sizeof and offsets of the three argument structs, from a C program."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {"nereus_logits_t": B.Logits, "nereus_penalties_t": B.Penalties, "nereus_distill_t": B.Distill}
    lines = []
    for name, cls in fields.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "nereus.h"\nint main(void) {' + "\n".join(lines) + "return 0;}")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    want = []
    for cls in fields.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f[0]).offset for f in cls._fields_]
    assert got == want


def test_the_torch_layer_refuses_host_tensors_and_wrong_types():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        L.process(x)
    with pytest.raises(ValueError):
        L.teacher_top(x.half(), 2)
    with pytest.raises(ValueError):
        L.distill_forward([x, x], torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))
