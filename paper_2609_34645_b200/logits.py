"""The model-stages' own steps on the LM head's logits, on torch tensors: ``process`` (generation), ``teacher_top``
(inference) and the distillation from a teacher's top logits (training), ``distill_forward`` / ``distill_backward`` /
``distill_step`` and, for autograd, ``distill_loss``.

Logits are one tensor [rows, vocab] or, where the head is cut over tensor-parallel ranks, the list of its column shards
[rows, shard_cols] in rank order; ``vocab`` says how many of the columns count when the vocabulary was padded before
the cut.  Shards are bf16 or fp32, contiguous along the vocabulary, all with the same stride between rows.

Everything runs in the CUDA library on torch's current stream and synchronises nothing; what is returned was allocated
on that stream unless the caller passed it in.  Wrong types, devices or shapes raise ValueError here, everything the
library refuses raises NereusError.
"""
from __future__ import annotations

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.BF16, torch.float32: B.FP32}
_DIVERGENCES = {"forward_kl": B.FORWARD_KL, "reverse_kl": B.REVERSE_KL, "js": B.JENSEN}


def _stream(device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _view(x, vocab, like=None):
    """(nereus_logits_t, first shard) of a tensor or a list of column shards."""
    shards = (x,) if isinstance(x, torch.Tensor) else x
    first = shards[0]
    if first.dim() != 2:
        raise ValueError("logits are [rows, columns] tensors")
    rows, cols = first.shape
    stride = first.stride(0) if rows > 1 else cols
    tp = len(shards)
    v = B.Logits()
    if tp > B.VOCAB_MAX_TP:
        raise ValueError(f"at most {B.VOCAB_MAX_TP} shards")
    dtype, device = first.dtype, first.device
    if dtype not in _DTYPES or device.type != "cuda":
        raise ValueError("logits are bf16 or fp32 tensors on a CUDA device")
    if like is not None and device != like.device:
        raise ValueError("read and written logits are on different devices")
    width = tp * cols if vocab is None else vocab
    ptr = v.shard
    for s, t in enumerate(shards):
        if s:
            if t.dtype != dtype or t.device != device or t.dim() != 2 or t.shape[0] != rows:
                raise ValueError("shards differ in type, device or rows")
            if t.shape[1] != cols:
                # the last shard of an unpadded cut of a trimmed vocabulary may be narrower
                if s + 1 < tp or vocab is None or t.shape[1] < min(cols, vocab - s * cols):
                    raise ValueError("shards differ in columns")
            if rows > 1 and t.stride(0) != stride:
                raise ValueError("shards differ in the stride between rows")
        if t.stride(1) != 1 and t.shape[1] > 1:
            raise ValueError("logits are contiguous along the vocabulary")
        ptr[s] = t.data_ptr()
    v.dtype, v.tp, v.rows, v.vocab, v.shard_cols, v.row_stride = _DTYPES[dtype], tp, rows, width, cols, stride
    return v, first


def _arg(t, dtype, shape, like, what):
    """Device address of an optional argument after its checks."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != like.device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {like.device}")
    return t.data_ptr()


def _empty_like(x, dtype=None):
    if isinstance(x, torch.Tensor):
        return torch.empty(x.shape, dtype=dtype or x.dtype, device=x.device)
    return [torch.empty(s.shape, dtype=dtype or s.dtype, device=s.device) for s in x]


def process(x, *, vocab=None, out=None, out_dtype=None, history=None, prompt_len=None, total_len=None, repetition=None,
            presence=None, frequency=None, bias_ids=None, bias_values=None, mask=None, mask_row=None):
    """(out, token, lse): penalties for repeated tokens, biases and grammar masks on a batch of rows; the greedy token
    (int32, -1 where nothing is allowed) and the log-sum-exp of every processed row.

    history [rows, n] int32: the prompt, then what was generated; prompt_len, total_len [rows] int32 (None: 0 and n).
    repetition, presence, frequency [rows] fp32.  bias_ids int32 / bias_values fp32 [rows, n].  mask [grammars, words]
    int32, token v in bit v % 32 of word v // 32; mask_row [rows] int32, -1 for none (None: mask r for row r).
    out: like x, in x's type or fp32 (default: new, of out_dtype); x itself processes in place."""
    src, first = _view(x, vocab)
    rows = src.rows
    if out is None:
        out = _empty_like(x, out_dtype)
    dst, _ = _view(out, src.vocab, first)
    row = (rows,)
    how = B.Penalties()
    if history is not None:
        if history.dtype != torch.int32 or history.dim() != 2 or history.shape[0] != rows or \
                history.device != first.device or (history.stride(1) != 1 and history.shape[1] > 1):
            raise ValueError("history: expected int32 [rows, n], contiguous along n, on the logits' device")
        if history.shape[1]:
            how.history = history.data_ptr()
            how.history_len = history.shape[1]
            how.history_stride = history.stride(0) if rows > 1 else history.shape[1]
            how.prompt_len = _arg(prompt_len, torch.int32, row, first, "prompt_len")
            how.total_len = _arg(total_len, torch.int32, row, first, "total_len")
    elif prompt_len is not None or total_len is not None:
        raise ValueError("prompt_len and total_len belong to a history")
    how.repetition = _arg(repetition, torch.float32, row, first, "repetition")
    how.presence = _arg(presence, torch.float32, row, first, "presence")
    how.frequency = _arg(frequency, torch.float32, row, first, "frequency")
    if bias_ids is not None and bias_ids.numel():
        how.bias_count = bias_ids.shape[-1]
        how.bias_ids = _arg(bias_ids, torch.int32, (rows, how.bias_count), first, "bias_ids")
        how.bias_values = _arg(bias_values, torch.float32, (rows, how.bias_count), first, "bias_values")
    if mask is not None:
        if mask.dtype != torch.int32 or mask.dim() != 2 or mask.device != first.device or \
                (mask.stride(1) != 1 and mask.shape[1] > 1) or mask.shape[1] * 32 < src.vocab:
            raise ValueError("mask: expected int32 [grammars, >= vocab / 32], contiguous along the words")
        how.mask, how.mask_rows = mask.data_ptr(), mask.shape[0]
        how.mask_stride = mask.stride(0) if mask.shape[0] > 1 else mask.shape[1]
        how.mask_row = _arg(mask_row, torch.int32, row, first, "mask_row")
    elif mask_row is not None:
        raise ValueError("mask_row belongs to a mask")
    token = torch.empty(row, dtype=torch.int32, device=first.device)
    lse = torch.empty(row, dtype=torch.float32, device=first.device)
    B.logits_process(src, dst, how, token.data_ptr(), lse.data_ptr(), _stream(first.device))
    return out, token, lse


def teacher_top(x, k, *, vocab=None, temperature=1.0):
    """(values fp32 [rows, k], ids int32 [rows, k], lse fp32 [rows]): a teacher's k largest logits, falling, equal ones
    by rising id, and the log-sum-exp of the row's logits / temperature."""
    src, first = _view(x, vocab)
    values = torch.empty((src.rows, k), dtype=torch.float32, device=first.device)
    ids = torch.empty((src.rows, k), dtype=torch.int32, device=first.device)
    lse = torch.empty((src.rows,), dtype=torch.float32, device=first.device)
    B.teacher_top(src, k, temperature, values.data_ptr(), ids.data_ptr(), lse.data_ptr(), _stream(first.device))
    return values, ids, lse


def _how(src, first, ids, values, lse, weight, divergence, temperature, beta):
    if divergence not in _DIVERGENCES:
        raise ValueError(f"divergence: one of {sorted(_DIVERGENCES)}")
    if ids.dim() != 2:
        raise ValueError("ids: expected int32 [rows, k]")
    k, rows = ids.shape[1], src.rows
    return B.Distill(k, _DIVERGENCES[divergence], beta, temperature,
                     _arg(values, torch.float32, (rows, k), first, "values"),
                     _arg(ids, torch.int32, (rows, k), first, "ids"), _arg(lse, torch.float32, (rows,), first, "lse"),
                     _arg(weight, torch.float32, (rows,), first, "weight"))


def distill_forward(x, ids, values, *, vocab=None, lse=None, weight=None, divergence="forward_kl", temperature=1.0,
                    beta=0.5):
    """(loss fp32 [rows], saved fp32 [rows, 4]): weight * the divergence of the student's logits x from a teacher's
    entries (ids int32, values fp32 [rows, k], as teacher_top returns them).  lse: the teacher's log-sum-exp at this
    temperature, so that what the entries leave is a group of its own; None renormalises the teacher over its entries
    (forward KL only).  weight fp32 [rows]: rows of weight 0 are not read.  divergence: "forward_kl", "reverse_kl", "js"
    (with beta).  saved goes to distill_backward: row maximum, sum of exp((x - max) / T), the same over the rest, D."""
    src, first = _view(x, vocab)
    how = _how(src, first, ids, values, lse, weight, divergence, temperature, beta)
    loss = torch.empty((src.rows,), dtype=torch.float32, device=first.device)
    saved = torch.empty((src.rows, 4), dtype=torch.float32, device=first.device)
    B.distill_forward(src, how, loss.data_ptr(), saved.data_ptr(), _stream(first.device))
    return loss, saved


def distill_backward(x, ids, values, saved, *, grad_loss=None, grad=None, vocab=None, lse=None, weight=None,
                     divergence="forward_kl", temperature=1.0, beta=0.5):
    """The gradient of sum(grad_loss * loss) with respect to x, in x's type and cut, from distill_forward's saved sums.
    grad: where to put it (default: new); x itself overwrites the logits.  Padding columns are not written."""
    src, first = _view(x, vocab)
    if grad is None:
        grad = _empty_like(x)
    dst, _ = _view(grad, src.vocab, first)
    how = _how(src, first, ids, values, lse, weight, divergence, temperature, beta)
    B.distill_backward(src, how, _arg(saved, torch.float32, (src.rows, 4), first, "saved"),
                       _arg(grad_loss, torch.float32, (src.rows,), first, "grad_loss"), dst, _stream(first.device))
    return grad


def distill_step(x, ids, values, *, grad=None, vocab=None, lse=None, weight=None, divergence="forward_kl",
                 temperature=1.0, beta=0.5):
    """(loss, grad) in one launch: distill_forward and the gradient of the sum of its losses, every logit read from
    memory once.  grad: where to put it (default: new); x itself overwrites the logits."""
    src, first = _view(x, vocab)
    if grad is None:
        grad = _empty_like(x)
    dst, _ = _view(grad, src.vocab, first)
    how = _how(src, first, ids, values, lse, weight, divergence, temperature, beta)
    loss = torch.empty((src.rows,), dtype=torch.float32, device=first.device)
    B.distill_step(src, how, loss.data_ptr(), dst, _stream(first.device))
    return loss, grad


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, values, how, *shards):
        x = shards[0] if len(shards) == 1 else list(shards)
        loss, saved = distill_forward(x, ids, values, **how)
        ctx.save_for_backward(ids, values, saved, *shards)
        ctx.how, ctx.n = how, len(shards)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        ids, values, saved, *shards = ctx.saved_tensors
        # columns past the vocabulary take no part in the loss
        padded = ctx.how["vocab"] is not None and ctx.how["vocab"] < sum(s.shape[1] for s in shards)
        new = torch.zeros if padded else torch.empty
        grad = [new(s.shape, dtype=s.dtype, device=s.device) for s in shards]
        x = shards[0] if ctx.n == 1 else shards
        distill_backward(x, ids, values, saved, grad_loss=grad_loss.contiguous(), grad=grad[0] if ctx.n == 1 else grad,
                         **ctx.how)
        return (None, None, None, *grad)


def distill_loss(x, ids, values, *, vocab=None, lse=None, weight=None, divergence="forward_kl", temperature=1.0,
                 beta=0.5):
    """distill_forward's loss [rows], differentiable with respect to x (a tensor or its shards)."""
    how = {"vocab": vocab, "lse": lse, "weight": weight, "divergence": divergence, "temperature": temperature, "beta": beta}
    return _DistillLoss.apply(ids, values, how, *((x,) if isinstance(x, torch.Tensor) else x))
