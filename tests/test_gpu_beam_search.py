"""A whole beam search over a paged cache (examples/beam_search.py), with forks, reordered states, a compaction on the way and copies
at the end, against one that keeps every hypothesis as a list of tokens and works everything out again in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def plain_search(example, model, prompt, beams, steps, penalty):
    """One request: lists of tokens, sorted never; returns the surviving hypotheses as (tokens, score, ended)."""
    alive = [(list(prompt), 0.0, False)]
    n = len(prompt)
    for _ in range(steps):
        offers = []
        for b, (tokens, score, ended) in enumerate(alive):
            made = len(tokens) - n
            if ended:
                offers.append((score / max(made, 1) ** 0.8, b, example.END, score, True))
                continue
            at = torch.arange(len(tokens), device="cuda")
            t = torch.tensor(tokens, device="cuda")
            keys, values = model.keys_and_values(t, at)
            x = torch.cat(model.logits(t[-1:], at[-1:], keys[None], values[None], at[-1:] + 1), 1)[0].cpu().numpy()
            seen = np.unique(tokens)
            x[seen] = np.where(x[seen] > 0, x[seen] / np.float32(penalty), x[seen] * np.float32(penalty))
            x = x.astype(np.float64)
            total = score + x - (np.log(np.exp(x - x.max()).sum()) + x.max())
            norm = np.float64(np.float32(max(made + 1, 1)) ** np.float32(0.8))
            offers += [(total[v] / norm, b, v, total[v], False) for v in np.argsort(-total)[:beams]]
        offers.sort(key=lambda o: -o[0])
        alive = [(alive[b][0] if was else alive[b][0] + [int(v)], s, was or v == example.END) for _, b, v, s, was in offers[:beams]]
    return alive


def test_a_search_over_a_paged_cache():
    import beam_search as example
    model, prompt, prompt_len, tokens, scores, left = example.main()
    beams, steps = tokens.shape[1:]
    for r in range(prompt.shape[0]):
        n = int(prompt_len[r])
        want = plain_search(example, model, prompt[r, :n].tolist(), beams, steps, 1.3)
        want = sorted((tuple(t[n:]), s) for t, s, _ in want)
        got = sorted((tuple(t[:t.index(example.END) + 1] if example.END in t else t), s) for t, s in zip(tokens[r].tolist(), scores[r].tolist()))
        assert [t for t, _ in got] == [t for t, _ in want]
        # 14 totals, each rounded to fp32 once and a sum of exponentials of 500 off by 2e-7 at most
        assert np.allclose([s for _, s in got], [s for _, s in want], rtol=0, atol=steps * (2e-7 + 2.0 ** -24 * 100))
    # what was copied to the other unit is the best beams' keys and values
    at = 0
    for r, (best, n) in enumerate(zip(left["best"].tolist(), left["length"].tolist())):
        history = torch.cat([prompt[r, :int(prompt_len[r])], tokens[r, best - r * beams]])[:n].long()
        keys, values = model.keys_and_values(history, torch.arange(n, device="cuda"))
        held = int(left["held"][r])
        for pool, want in zip(left["other"], (keys, values)):
            # products of another shape may round otherwise
            assert torch.allclose(pool[at:at + held].reshape(-1, example.HIDDEN)[:n], want, rtol=0, atol=1e-12)
        at += held
    table, length, refs = left["books"]
    assert (table == -1).all() and (length == 0).all()
    assert set(refs.tolist()) <= {0, 1} and int((refs == 0).sum()) >= 3 * beams * 6      # only what was given away is still held
