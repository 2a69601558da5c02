"""A generation stage's beam search over a paged cache, in small, with the calls of ``logits`` and ``cache``:

  prompt        one row per request writes its keys and values into pages
  first step    every request's row is forked into its beams: full pages are shared, the begun one is copied
  each step     process (a repetition penalty on the cut logits), beam_select (ended beams among them, ranked by length),
                fork (the cache follows the beams that go on, with room for the next token) and reorder (so do the token
                history and what else a program keeps per row)
  half way      compact: the pages in use move to the front, and the search goes on in the pools' first pages alone, as when a
                plan transition needs the memory behind them
  at the end    copy: the best beams' pages go to another unit's cache; fork to no rows at all frees the rest

The decoder is one attention layer over random weights, in torch.  Run on a B200:

  python examples/beam_search.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_34645_b200 import cache as C                        # noqa: E402
from paper_2609_34645_b200 import logits as L                       # noqa: E402

VOCAB, HIDDEN, TP, PAGE, PAGES = 500, 32, 2, 4, 160
END = 7                                                             # the token that ends an answer


class Decoder:
    """One layer of attention; keys and values of a token depend on the token and its position alone."""

    def __init__(self, device="cuda", seed=0):
        gen = torch.Generator(device).manual_seed(seed)
        rand = lambda *n: torch.randn(*n, generator=gen, device=device, dtype=torch.float64)        # noqa: E731
        self.embed, self.place = rand(VOCAB, HIDDEN), rand(256, HIDDEN)
        self.key, self.value, self.query = rand(HIDDEN, HIDDEN) / 6, rand(HIDDEN, HIDDEN) / 3, rand(HIDDEN, HIDDEN) / 6
        self.head = list((rand(VOCAB, HIDDEN) / 3).split(VOCAB // TP))                               # cut over the ranks

    def keys_and_values(self, token, at):
        h = self.embed[token] + self.place[at]
        return h @ self.key, h @ self.value

    def logits(self, token, at, keys, values, length):
        """The next token's logits, a shard per rank: `keys`, `values` [rows, n, hidden], of which length[row] count."""
        h = self.embed[token] + self.place[at]
        weight = torch.einsum("rd,rnd->rn", h @ self.query, keys)
        behind = torch.arange(keys.shape[1], device=keys.device) >= length[:, None]
        weight = weight.masked_fill(behind, -torch.inf)
        h = h + torch.einsum("rn,rnd->rd", weight.softmax(1), values.masked_fill(behind[:, :, None], 0.0))
        return [(h @ w.T).float() for w in self.head]


def put(pools, table, row_length, model, token):
    """Writes one more token of every row behind its length."""
    at = row_length.long()
    page = table.gather(1, (at // PAGE)[:, None])[:, 0].long()
    for pool, new in zip(pools, model.keys_and_values(token, at)):
        pool[page, at % PAGE] = new
    return row_length + 1


def search(model, prompt, prompt_len, beams=4, steps=14, penalty=1.3, device="cuda"):
    """(tokens [requests, beams, steps], scores [requests, beams], what is left of the cache)."""
    requests = prompt.shape[0]
    columns = -(-(int(prompt_len.max()) + steps + 1) // PAGE)
    pools = [torch.zeros(PAGES, PAGE, HIDDEN, device=device, dtype=torch.float64) for _ in range(2)]
    ints = lambda *n, fill=0: torch.full(n, fill, dtype=torch.int32, device=device)                 # noqa: E731
    books = (ints(requests, columns, fill=-1), ints(requests), ints(PAGES))
    itself = torch.arange(requests, dtype=torch.int32, device=device)

    # the prompt but for its last token, by rows
    *books, _, _ = C.fork(pools, *books, itself, PAGE, room=prompt_len)
    for j in range(prompt.shape[1]):
        more = j < prompt_len - 1
        grown = put(pools, books[0], books[1], model, prompt[:, j])  # what stands behind a row's length is overwritten
        books[1] = torch.where(more, grown, books[1])

    # every request's row becomes its beams; all but the first offer nothing on the first step
    parent = itself.repeat_interleave(beams)
    *books, _, status = C.fork(pools, *books, parent, PAGE, room=1)
    history = torch.cat([prompt, ints(requests, steps)], 1).repeat_interleave(beams, 0)
    total = prompt_len.repeat_interleave(beams)
    token = prompt.gather(1, prompt_len[:, None].long() - 1)[:, 0].repeat_interleave(beams)
    score = torch.where(torch.arange(requests * beams, device=device) % beams == 0, 0.0, -torch.inf)
    ended = ints(requests * beams, fill=-1)
    rho = torch.full((requests * beams,), penalty, device=device)
    made = ints(requests * beams)                                   # tokens of the answer
    for step in range(steps):
        on = ended < 0
        length = put(pools, books[0], books[1], model, token)
        books[1] = torch.where(on, length, books[1])                # an ended beam's cache stays as it is
        table, n = books[0].clamp(min=0).long(), columns * PAGE
        keys, values = (p[table].view(-1, n, HIDDEN) for p in pools)
        x = model.logits(token, length.long() - 1, keys, values, length)
        L.process(x, vocab=VOCAB, out=x, history=history, total_len=total, repetition=rho)
        norm = (made + on).clamp(min=1).float() ** 0.8
        score, parent, token = (t.view(-1) for t in L.beam_select(x, score, beams, beams=beams, vocab=VOCAB, ended=ended, norm=norm, settle=True))
        # everything that a row has follows its beam
        *books, _, status = C.fork(pools, *books, parent, PAGE, room=1)
        for state in (history, total, made, ended):
            C.reorder(state, parent, beams=beams)
        on = ended < 0
        history.scatter_(1, total[:, None].long(), torch.where(on, token, history.gather(1, total[:, None].long())[:, 0])[:, None])
        total, made = total + on, made + on
        ended = torch.where(on & (token == END), END, ended)
        if step == steps // 2:
            table, refs, _, _, status = C.compact(pools, books[0], books[2])
            keep = int(status[3])
            for p in pools:                                         # what lies behind is somebody else's now
                p[keep:] = torch.nan
            refs[min(PAGES, keep + requests * beams * 6):] = 1
            books[0], books[2] = table, refs
    # the best beam of every request goes to another unit
    best = (score / made.clamp(min=1) ** 0.8).view(requests, beams).argmax(1) + beams * torch.arange(requests, device=device)
    src = books[0][best]
    held = src >= 0
    other = [torch.zeros_like(p) for p in pools]
    C.copy(pools, src[held], torch.arange(int(held.sum()), dtype=torch.int32, device=device), to=other)
    length, books = books[1][best], C.fork(pools, *books, ints(requests * beams, fill=-1), PAGE)[:3]
    answers = torch.stack([h[n:n + steps] for h, n in zip(history, prompt_len.repeat_interleave(beams).tolist())])
    return answers.view(requests, beams, steps), score.view(requests, beams), {
        "books": books, "other": other, "held": held.sum(1), "length": length, "best": best}


def main(device="cuda"):
    gen = torch.Generator(device).manual_seed(1)
    prompt_len = torch.tensor([9, 5, 12], dtype=torch.int32, device=device)
    prompt = torch.randint(VOCAB, (3, 12), generator=gen, device=device, dtype=torch.int32)
    model = Decoder(device)
    return model, prompt, prompt_len, *search(model, prompt, prompt_len, device=device)


if __name__ == "__main__":
    _, _, _, tokens, scores, _ = main()
    for r, (answers, score) in enumerate(zip(tokens.tolist(), scores.tolist())):
        for a, s in sorted(zip(answers, score), key=lambda t: -t[1]):
            print(f"request {r}: {s:8.3f}  {a}")
