"""The model-stages' own steps on the LM head's logits, on torch tensors: ``process`` and ``beam_select`` (generation),
``teacher_top`` (inference) and the distillation from a teacher's top logits (training), ``distill_forward`` / ``distill_backward`` /
``distill_step`` and, for autograd, ``distill_loss``.

Logits are one tensor [rows, vocab] or, where the head is cut over tensor-parallel ranks, the list of its column shards
[rows, shard_cols] in rank order; ``vocab`` says how many of the columns count when the vocabulary was padded before
the cut, or the last shard is narrower than the others.  Shards are bf16 or fp32, contiguous along the vocabulary, all with
the same stride between rows (a narrower last one, as ``x.split(w, dim=1)`` gives it, is a slice of the same tensor).

Everything runs in the CUDA library on torch's current stream and synchronises nothing; what is returned was allocated
on that stream unless the caller passed it in.  Wrong types, devices or shapes raise ValueError, everything the library
refuses raises NereusError.  Under autograd only ``distill_loss`` is differentiable; what the other calls return carries no
gradient, whatever the logits require.  The arguments are marshalled by ``_nereus_torch.so`` (``python -m
paper_2609_34645_b200.build``); importing this module without it raises.
"""
from __future__ import annotations

import torch

from . import binding as B

try:
    from . import _nereus_torch as _t
except ImportError as e:
    raise ImportError("_nereus_torch.so is missing or does not load: build it with `python -m "
                      "paper_2609_34645_b200.build`") from e

_t.set_error(B.NereusError)
_DIVERGENCES = {"forward_kl": B.FORWARD_KL, "reverse_kl": B.REVERSE_KL, "js": B.JENSEN}


def _divergence(name):
    if name not in _DIVERGENCES:
        raise ValueError(f"divergence: one of {sorted(_DIVERGENCES)}")
    return _DIVERGENCES[name]


def process(x, *, vocab=None, out=None, out_dtype=None, history=None, prompt_len=None, total_len=None, repetition=None,
            presence=None, frequency=None, bias_ids=None, bias_values=None, mask=None, mask_row=None):
    """(out, token, lse): penalties for repeated tokens, biases and grammar masks on a batch of rows; the greedy token
    (int32, -1 where nothing is allowed) and the log-sum-exp of every processed row.

    history [rows, n] int32: the prompt, then what was generated; prompt_len, total_len [rows] int32 (None: 0 and n).
    repetition, presence, frequency [rows] fp32.  bias_ids int32 / bias_values fp32 [rows, n].  mask [grammars, words]
    int32, token v in bit v % 32 of word v // 32; mask_row [rows] int32, -1 for none (None: mask r for row r).
    out: like x, in x's type or fp32 (default: new, of out_dtype); x itself processes in place."""
    return _t.process(x, vocab, out, out_dtype, history, prompt_len, total_len, repetition, presence, frequency, bias_ids,
                      bias_values, mask, mask_row)


def beam_select(x, score, k, *, beams, vocab=None, ended=None, norm=None, settle=False):
    """(score fp32, parent int32, token int32), each [requests, k]: one step of a beam search.  x has requests * beams rows;
    of all hypotheses score + x - logsumexp(x) of a request's beams the k best, falling, equal ones by rising beam and
    token.  parent is the row that a hypothesis goes on from, for ``cache.reorder`` and ``cache.fork``; places for which
    nothing is left get (-inf, -1, -1).

    score [rows] fp32: of the beams so far; a beam of -inf offers nothing (and all but a request's first do on its first
    step).  ended [rows] int32: the token of a beam that has ended, which offers itself alone, -1 for one that goes on.
    norm [rows] fp32 > 0: hypotheses are ranked by score / norm, as by their lengths.  settle (k == beams): the best that
    goes on from a row is put at that row's place, so that only rows that nothing goes on from are overwritten."""
    return _t.beam_select(x, vocab, score, k, beams, ended, norm, settle)


def teacher_top(x, k, *, vocab=None, temperature=1.0):
    """(values fp32 [rows, k], ids int32 [rows, k], lse fp32 [rows]): a teacher's k largest logits, falling, equal ones
    by rising id, and the log-sum-exp of the row's logits / temperature."""
    return _t.teacher_top(x, k, vocab, temperature)


def distill_forward(x, ids, values, *, vocab=None, lse=None, weight=None, divergence="forward_kl", temperature=1.0,
                    beta=0.5):
    """(loss fp32 [rows], saved fp32 [rows, 4]): weight * the divergence of the student's logits x from a teacher's
    entries (ids int32, values fp32 [rows, k], as teacher_top returns them).  lse: the teacher's log-sum-exp at this
    temperature, so that what the entries leave is a group of its own; None renormalises the teacher over its entries
    (forward KL only).  weight fp32 [rows]: rows of weight 0 are not read.  divergence: "forward_kl", "reverse_kl", "js"
    (with beta).  saved goes to distill_backward: row maximum, sum of exp((x - max) / T), the same over the rest, D."""
    return _t.distill_forward(x, vocab, ids, values, lse, weight, _divergence(divergence), temperature, beta)


def distill_backward(x, ids, values, saved, *, grad_loss=None, grad=None, vocab=None, lse=None, weight=None,
                     divergence="forward_kl", temperature=1.0, beta=0.5):
    """The gradient of sum(grad_loss * loss) with respect to x, in x's type and cut, from distill_forward's saved sums.
    grad: where to put it (default: new); x itself overwrites the logits.  Padding columns are not written."""
    return _t.distill_backward(x, vocab, ids, values, lse, weight, _divergence(divergence), temperature, beta, saved,
                               grad_loss, grad)


def distill_step(x, ids, values, *, grad=None, vocab=None, lse=None, weight=None, divergence="forward_kl",
                 temperature=1.0, beta=0.5):
    """(loss, grad) in one launch: distill_forward and the gradient of the sum of its losses.  grad: where to put it
    (default: new); x itself overwrites the logits."""
    return _t.distill_step(x, vocab, ids, values, lse, weight, _divergence(divergence), temperature, beta, grad)


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, values, lse, weight, how, *shards):
        x = shards[0] if len(shards) == 1 else list(shards)
        loss, saved = distill_forward(x, ids, values, lse=lse, weight=weight, **how)
        ctx.save_for_backward(ids, values, lse, weight, saved, *shards)
        ctx.how, ctx.n = how, len(shards)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        ids, values, lse, weight, saved, *shards = ctx.saved_tensors
        grad = _t.empty_like(shards)
        # columns past the vocabulary take no part in the loss
        if ctx.how["vocab"] is not None and ctx.how["vocab"] < sum(s.shape[1] for s in shards):
            for g in grad:
                g.zero_()
        x = shards[0] if ctx.n == 1 else shards
        distill_backward(x, ids, values, saved, grad_loss=grad_loss.contiguous(), grad=grad[0] if ctx.n == 1 else grad,
                         lse=lse, weight=weight, **ctx.how)
        return (None, None, None, None, None, *grad)


def distill_loss(x, ids, values, *, vocab=None, lse=None, weight=None, divergence="forward_kl", temperature=1.0,
                 beta=0.5):
    """distill_forward's loss [rows], differentiable with respect to x (a tensor or its shards) and to nothing else: the
    teacher's side and the weights may not require a gradient."""
    for name, t in (("values", values), ("lse", lse), ("weight", weight)):
        if isinstance(t, torch.Tensor) and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name}: distill_loss has no gradient with respect to it; detach it")
    how = {"vocab": vocab, "divergence": divergence, "temperature": temperature, "beta": beta}
    return _DistillLoss.apply(ids, values, lse, weight, how, *((x,) if isinstance(x, torch.Tensor) else x))
