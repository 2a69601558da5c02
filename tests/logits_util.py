"""Helpers of the tests of the steps on an LM head's logits: cuts of a logical [rows, vocab] array into column shards of
several memory layouts, written views with a sentinel around them, and the definitions in 64 bits (numpy)."""
from __future__ import annotations

import numpy as np
import torch

SENTINEL = -77.0
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 2.0 ** -24          # half a unit in the last place of fp32, relative


def width(vocab, tp, padded):
    """Columns per shard: the even cut, or the cut of the vocabulary padded to a multiple of 128 * tp."""
    return -(-vocab // (128 * tp)) * 128 if padded else -(-vocab // tp)


class View:
    """[rows, vocab] logits cut over tp shards in one of the layouts
        "shards"   every shard a contiguous tensor of its own
        "columns"  column slices of one tensor
        "odd"      column slices of a wider tensor that starts one element in: no row is 16-byte aligned as a rule
    with everything outside the logical columns set to `fill`."""

    def __init__(self, rows, vocab, tp, dtype, layout, padded=False, fill=float("nan")):
        self.rows, self.vocab, self.tp, self.w = rows, vocab, tp, width(vocab, tp, padded)
        full = self.w * tp
        dt = TYPES[dtype]
        if layout == "shards":
            self.raw = [torch.full((rows, self.w), fill, dtype=dt, device="cuda") for _ in range(tp)]
            self.shards = self.raw
        else:
            extra, start = (0, 0) if layout == "columns" else (5, 1)
            whole = torch.full((rows * (full + extra) + 16,), fill, dtype=dt, device="cuda")
            self.raw = [whole]
            self.shards = [torch.as_strided(whole, (rows, self.w), (full + extra, 1), start + s * self.w)
                           for s in range(tp)]
        self.fill = fill

    def put(self, x):
        """x: [rows, vocab] tensor, rounded to the view's type."""
        for s, shard in enumerate(self.shards):
            part = x[:, s * self.w:min((s + 1) * self.w, self.vocab)]
            shard[:, :part.shape[1]] = part.to(shard.dtype).to(shard.device)
        return self

    def get(self):
        return torch.cat(self.shards, dim=1)[:, :self.vocab]

    def arg(self):
        return self.shards[0] if self.tp == 1 else self.shards

    def untouched_outside(self):
        """Whether every element outside the logical columns still holds the fill."""
        keep = [r.clone() for r in self.raw]
        self.put(torch.full((self.rows, self.vocab), self.fill))
        ok = all(bool((r == self.fill).all()) for r in self.raw)
        for r, k in zip(self.raw, keep):
            r.copy_(k)
        return ok


def rounded(x, dtype):
    """float64 values of x after rounding to the type."""
    return torch.as_tensor(x).to(TYPES[dtype]).double().cpu().numpy()


def log_sum_exp(x):
    with np.errstate(all="ignore"):
        m = x.max(axis=1)
        safe = np.where(np.isfinite(m), m, 0.0)
        s = np.log(np.exp(x - safe[:, None]).sum(axis=1)) + safe
    return np.where(np.isnan(x).any(axis=1), np.nan, np.where(np.isinf(m), m, s))


def sum_error(vocab):
    """Bound of the relative error of a sum of `vocab` positive exponentials in fp32 when at least 128 partial sums are
    kept: the longest partial sum, the joining of them, and the exponential's own two units."""
    return (vocab / 128 + 64) * EPS


def distill_definition(x, ids, values, lse, temperature, divergence, beta):
    """(D [rows], dD/dx [rows, vocab], sums [rows, 4]) in 64 bits; entries with ids outside the vocabulary unused."""
    rows, vocab = x.shape
    d, grad, sums = np.zeros(rows), np.zeros((rows, vocab)), np.zeros((rows, 4))
    with np.errstate(all="ignore"):
        for r in range(rows):
            use = (ids[r] >= 0) & (ids[r] < vocab)
            at, y = ids[r][use], values[r][use] / temperature
            m = x[r].max()
            e = np.exp((x[r] - m) / temperature)
            total = e.sum()
            rest_of = np.ones(vocab, bool)
            rest_of[at] = False
            rest = e[rest_of].sum()
            q = np.append(e[at], rest) / total
            if lse is None:
                p = np.exp(y - y.max()) if len(y) else y
                p = np.append(p / p.sum() if len(y) else y, 0.0)
                mass = 1.0 if len(y) else 0.0
            else:
                p = np.exp(y - lse[r])
                p = np.append(p, max(0.0, 1 - p.sum()) if rest_of.any() else 0.0)
                mass = 1.0
            group = np.full(vocab, len(at))
            group[at] = np.arange(len(at))
            if divergence == "forward_kl":
                d[r] = np.where(p > 0, p * np.log(p / q), 0).sum()
                qf = -p
                slope = np.where(p > 0, -p / q, 0.0)
                grad[r] = e / total * (slope[group] + mass)
                grad[r][at] = mass * q[:-1] - p[:-1]                # finite where q is 0
            else:
                if divergence == "reverse_kl":
                    p[-1] = max(p[-1], 2.0 ** -24)
                    slope = np.where(q > 0, np.log(q / p), 0.0)
                    d[r] = (q * slope).sum()
                else:
                    mix = beta * p + (1 - beta) * q
                    slope = np.where(q > 0, (1 - beta) * np.log(q / mix), 0.0)
                    d[r] = (q * slope).sum() + np.where(p > 0, beta * p * np.log(p / mix), 0).sum()
                qf = q * slope
                grad[r] = e / total * (slope[group] - qf.sum())
            sums[r] = m, total, rest, d[r]
    return d, grad / temperature, sums


def process_definition(x, how):
    """The processed row in fp32, every step rounded on its own (numpy float32 arithmetic rounds each operation).
    x: float32 [rows, vocab]; how: dict of numpy arrays."""
    x = x.astype(np.float32).copy()
    rows, vocab = x.shape
    one = np.ones(rows, np.float32)
    rho, pres, freq = how.get("repetition", one), how.get("presence", 0 * one), how.get("frequency", 0 * one)
    with np.errstate(all="ignore"):
        for r in range(rows):
            if "history" in how:
                h = how["history"][r]
                n = int(np.clip(how["total_len"][r] if "total_len" in how else len(h), 0, len(h)))
                a = int(how["prompt_len"][r]) if "prompt_len" in how else 0
                inside = [(j, t) for j, t in enumerate(h[:n]) if 0 <= t < vocab]
                for t in {t for _, t in inside}:
                    x[r, t] = x[r, t] / rho[r] if x[r, t] > 0 else x[r, t] * rho[r]
                    made = sum(1 for j, u in inside if u == t and j >= a)
                    if made:
                        x[r, t] = (x[r, t] - freq[r] * np.float32(made)) - pres[r]
            if "bias_ids" in how:
                last = {int(t): b for t, b in zip(how["bias_ids"][r], how["bias_values"][r]) if 0 <= t < vocab}
                for t, b in last.items():
                    x[r, t] = x[r, t] + b
            if "mask" in how:
                g = int(how["mask_row"][r]) if "mask_row" in how else r
                if 0 <= g < len(how["mask"]):
                    v = np.arange(vocab)
                    bits = how["mask"][g].astype(np.int64)[v >> 5] >> (v & 31) & 1
                    x[r, bits == 0] = -np.inf
    return x
