"""Cases for measuring what a generation stage does after its logits: ``logits.beam_select`` (of the beams of a request
times the vocabulary the k best hypotheses), ``cache.reorder`` (the rows of dense states follow the beams that go on) and,
where a cache is paged, ``cache.fork`` (page table, lengths and reference counts follow: full pages are shared, partly
filled ones copied, dropped ones freed, room is made for new tokens), ``cache.compact`` (pages in use move to the front of
the pools) and ``cache.copy`` (pages to other pages, or to another cache).

Logits are rows x vocabulary, cut into `tp` column shards; where the vocabulary does not divide, it is padded to a multiple
of 128 * tp first and the padding columns hold NaN, which nothing may read as a value.  States and pools are one tensor
here, of which a program's buffers are slices.

`run` computes them with elementary torch operations (``own`` false) or through ``paper_2609_34645_b200`` (``own`` true);
`exact` gives a selection's scores in 64 bits.  What the others return was moved, not computed.
"""
import math

import torch

own = False

BF16, FP32, INT8 = "bf16", "fp32", "int8"
TYPES = {BF16: torch.bfloat16, FP32: torch.float32, INT8: torch.int8}
INF = math.inf


# ---- the cases -------------------------------------------------------------------------------------------------

def _select(name, requests, beams, vocab, tp, dtype, k, ended, dead, norm, settle):
    return {"name": name, "op": "select", "requests": requests, "beams": beams, "vocab": vocab, "tp": tp, "dtype": dtype,
            "k": k, "ended": ended, "dead": dead, "norm": norm, "settle": settle}


def _reorder(name, buffers, from_rows, requests, beams, tokens, heads, width, dtype, place, heads_first):
    return {"name": name, "op": "reorder", "buffers": buffers, "from_rows": from_rows, "requests": requests, "beams": beams,
            "tokens": tokens, "heads": heads, "width": width, "dtype": dtype, "in_place": place, "heads_first": heads_first}


def _fork(name, requests, beams, shortest, longest, page_size, pools, width, dtype, spare, kept, freed, room):
    return {"name": name, "op": "fork", "requests": requests, "beams": beams, "shortest": shortest, "longest": longest,
            "page_size": page_size, "pools": pools, "width": width, "dtype": dtype, "spare": spare, "kept": kept,
            "freed": freed, "room": room}


def _compact(name, rows, columns, pages, live, keep, pools, page, dtype):
    return {"name": name, "op": "compact", "rows": rows, "columns": columns, "pages": pages, "live": live, "keep": keep,
            "pools": pools, "page": page, "dtype": dtype}


def _copy(name, pages, pairs, pools, page, dtype, other):
    return {"name": name, "op": "copy", "pages": pages, "pairs": pairs, "pools": pools, "page": page, "dtype": dtype,
            "other": other}


def listed():
    return [
        # one request that decodes alone with four beams: latency is all that counts
        _select("select 1 x 4", 1, 4, 128256, 1, BF16, 8, 0, 0, False, False),
        # a decode step of 128 requests with eight beams, head over 4 ranks, some beams at their end, some not started
        _select("select 128 x 8 tp4", 128, 8, 128256, 4, BF16, 16, 80, 112, True, False),
        # an odd vocabulary in fp32, odd beams; the beams that go on keep their rows
        _select("select 37 x 5 odd", 37, 5, 50257, 1, FP32, 5, 11, 0, True, True),
        # the dense cache of 16 of the 8B model's layers, TP4, 8 requests of 8 beams at every stage of their answers
        _reorder("reorder 64 rows", 32, 64, 8, 8, 2048, 2, 128, BF16, True, False),
        # a short prompt's states handed from its one row to the request's four beams, all 32 layers
        _reorder("reorder 1 to 4", 64, 1, 1, 4, 300, 2, 128, BF16, False, True),
        # one request of four beams, all 32 layers
        _fork("fork 4 rows", 1, 4, 900, 900, 16, 64, 256, BF16, 100, 0, 0, 1),
        # 16 requests of eight beams, all 32 layers, TP4
        _fork("fork 128 rows", 16, 8, 40, 2040, 16, 64, 256, BF16, 400, 0, 1, 1),
        # a server's batch: long contexts, most rows go on alone, some are sampled from twice, some are done
        _fork("fork 1024 rows long", 512, 2, 700, 32000, 16, 2, 64, BF16, 4000, 400, 40, 1),
        # before a change of plan: the pages in use, two in five, to the front, and the rest of the pools handed back
        _compact("compact 6000 pages", 128, 129, 6000, 2400, -1, 64, 4096, BF16),
        # a small odd cache of one byte an element, cut to a given size
        _compact("compact 257 pages odd", 7, 31, 257, 120, 200, 4, 13 * 45, INT8),
        # 700 pages of all 32 layers, TP4, to a replica's cache
        _copy("copy 700 pages", 4000, 700, 64, 4096, BF16, True),
        # a handful of pages
        _copy("copy 5 pages odd", 100, 5, 6, 13 * 45, INT8, False),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["select", "select", "select", "reorder", "reorder", "fork", "fork", "compact", "copy"])
    if op == "select":
        vocab = rng.choice([128256, 152064, 50257, _spread(rng, 8000, 160000), _spread(rng, 8000, 160000) | 1])
        beams = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
        dtype = rng.choice([BF16, BF16, FP32])
        requests = _spread(rng, 1, max(1, min(256, 200_000_000 // (vocab * beams * _size(dtype)))))
        settle = rng.random() < 0.3
        rows = requests * beams
        ended = rng.choice([0, rng.randint(0, rows // 3)])
        return {"op": op, "requests": requests, "beams": beams, "vocab": vocab, "tp": rng.choice([1, 1, 2, 4, 8]),
                "dtype": dtype, "k": beams if settle else rng.choice([beams, 2 * beams]),
                "ended": ended, "dead": rng.choice([0, rng.randint(0, rows // 3)]), "norm": rng.random() < 0.5,
                "settle": settle}
    dtype = rng.choice([BF16, BF16, FP32, INT8])
    if op == "reorder":
        beams, requests = rng.choice([2, 3, 4, 8, 12, 32]), _spread(rng, 1, 16)
        heads, width = rng.choice([1, 2, 3, 8]), rng.choice([64, 96, 128, 50])
        buffers = rng.choice([1, 2, 16, 64])
        tokens = _spread(rng, 1, min(4096, max(2, 1_000_000_000 // (beams * requests * heads * width * buffers * _size(dtype)))))
        place = rng.random() < 0.6
        return {"op": op, "buffers": buffers, "from_rows": beams * requests if place else _spread(rng, 1, beams * requests),
                "requests": requests, "beams": beams, "tokens": tokens, "heads": heads, "width": width, "dtype": dtype,
                "in_place": place, "heads_first": rng.random() < 0.5}
    pools, width = rng.choice([1, 2, 16, 64]), rng.choice([64, 128, 256, 45])
    if op == "fork":
        beams, requests = rng.choice([1, 2, 4, 8, 16]), _spread(rng, 1, 128)
        page_size = rng.choice([8, 16, 32, 64, 13])
        longest = _spread(rng, 1, max(2, min(32000, 1_500_000_000 // (pools * width * beams * requests * _size(dtype)))))
        kept = rng.choice([0, 0, requests // 2, requests])
        return {"op": op, "requests": requests, "beams": beams, "shortest": max(1, longest // rng.choice([1, 3, 50])),
                "longest": longest, "page_size": page_size, "pools": pools, "width": width, "dtype": dtype,
                "spare": rng.choice([requests * beams, 0, 300]), "kept": kept,
                "freed": rng.randint(0, (requests - kept) // 4), "room": rng.choice([0, 1, 1, 40])}
    page = width * rng.choice([8, 16, 13])
    pages = _spread(rng, 20, max(40, min(100_000, 1_200_000_000 // (pools * page * _size(dtype)))))
    if op == "copy":
        return {"op": op, "pages": pages, "pairs": _spread(rng, 1, pages // 2), "pools": pools, "page": page, "dtype": dtype,
                "other": rng.random() < 0.4}
    live = rng.randint(1, pages - 1)
    return {"op": op, "rows": _spread(rng, 1, 512), "columns": _spread(rng, 1, 500), "pages": pages, "live": live,
            "keep": rng.choice([-1, -1, rng.randint(live, pages)]), "pools": pools, "page": page, "dtype": dtype}


def _size(dtype):
    return {BF16: 2, FP32: 4, INT8: 1}[dtype]


def _lengths(case, count, low, high):
    """Lengths from `low` to `high`, evenly spread; the seed only deals them out."""
    return [low + (high - low) * i // max(1, count - 1) for i in range(count)]


def _survivors(beams):
    return (beams + 1) // 2


def work(case):
    op = case["op"]
    if op == "select":
        rows, v = case["requests"] * case["beams"], case["vocab"]
        live = max(0, rows - case["ended"] - case["dead"])
        per_row = 4 + 4 + 4 * case["norm"]
        return {"bytes": live * v * _size(case["dtype"]) + rows * per_row + case["requests"] * case["k"] * 12,
                "flops": live * v * 4}
    if op == "reorder":
        token = case["heads"] * case["width"] * _size(case["dtype"]) * case["buffers"]
        rows, b = case["requests"] * case["beams"], case["beams"]
        if case["in_place"]:
            total = sum(_lengths(case, case["requests"], max(1, case["tokens"] // 4), case["tokens"]))
            moved = b - _survivors(b)
            return {"bytes": total * token * (min(moved, _survivors(b)) + moved) + rows * 8, "flops": 0}
        lengths = _lengths(case, case["from_rows"], max(1, case["tokens"] // 4), case["tokens"])
        read = min(rows, case["from_rows"])
        mean = sum(lengths) / len(lengths)
        return {"bytes": int(mean * token * (read + rows)) + rows * 8, "flops": 0}
    if op == "fork":
        page = case["page_size"] * case["width"] * _size(case["dtype"]) * case["pools"]
        lengths = _lengths(case, case["requests"], case["shortest"], case["longest"])
        share = (case["requests"] - case["kept"] - case["freed"]) / case["requests"]
        copies = share * sum(n % case["page_size"] > 0 for n in lengths) * (case["beams"] - _survivors(case["beams"]))
        entries = sum(-(-n // case["page_size"]) for n in lengths) * case["beams"]
        tables = 4 * entries + 4 * _columns(case) * case["requests"] * case["beams"]
        return {"bytes": int(copies * 2 * page) + tables + 8 * _pages(case) + 12 * case["requests"] * case["beams"],
                "flops": 0}
    page = case["page"] * _size(case["dtype"]) * case["pools"]
    if op == "copy":
        return {"bytes": case["pairs"] * (2 * page + 8), "flops": 0}
    keep = case["live"] if case["keep"] < 0 else case["keep"]
    moved = case["live"] * (1 - keep / case["pages"])
    return {"bytes": int(moved * 2 * page) + 8 * case["rows"] * case["columns"] + 12 * case["pages"], "flops": 0}


# ---- the inputs ------------------------------------------------------------------------------------------------

def _logits(gen, rows, vocab):
    """Rows as a language model gives them: a broad bulk, and a few dozen tokens that stand out of it."""
    x = torch.randn(rows, vocab, generator=gen, device="cuda").mul_(1.6)
    few = min(40, vocab)
    part = vocab // few
    at = torch.randint(part, (rows, few), generator=gen, device="cuda") + part * torch.arange(few, device="cuda")
    lift = torch.empty(rows, few, device="cuda").exponential_(0.35, generator=gen).add_(4.0)
    return x.scatter_(1, at, lift)


def _cut(x, case):
    """The column shards, each a tensor of its own; padding columns are NaN."""
    v, tp = case["vocab"], case["tp"]
    w = v // tp if v % tp == 0 else -(-v // (128 * tp)) * 128
    whole = torch.nn.functional.pad(x, (0, w * tp - v), value=math.nan)
    return [s.to(TYPES[case["dtype"]]).contiguous() for s in whole.split(w, dim=1)]


def _fill(gen, shape, dtype):
    if dtype == INT8:
        return torch.randint(-128, 128, shape, generator=gen, device="cuda", dtype=torch.int8)
    return torch.empty(shape, dtype=TYPES[dtype], device="cuda").normal_(generator=gen)


def _shuffled(gen, n):
    return torch.randperm(n, generator=gen, device="cuda")


def _parents(gen, requests, beams, settled):
    """For every beam of every request the row that it goes on from: about half of a request's beams do, and the others'
    rows are taken by copies of them; settled: who goes on stays where it was."""
    order = torch.rand(requests, beams, generator=gen, device="cuda").argsort(1)
    take = order.gather(1, (torch.arange(beams, device="cuda") % _survivors(beams)).expand(requests, beams))
    if settled:
        local = torch.empty_like(order).scatter_(1, order, take)
    else:
        local = take.gather(1, torch.rand(requests, beams, generator=gen, device="cuda").argsort(1))
    return (local + beams * torch.arange(requests, device="cuda")[:, None]).int().view(-1)


def _columns(case):
    return -(-(case["longest"] + case["room"]) // case["page_size"])


def _pages(case):
    """Pages of the pools: what the sequences hold when half of each request's pages are its beams' common ones."""
    held = 0
    for n in _lengths(case, case["requests"], case["shortest"], case["longest"]):
        both = -(-n // case["page_size"])
        common = n // case["page_size"] // 2
        held += common + case["beams"] * (both - common)
    return held + case["requests"] * case["beams"] * (1 + -(-case["room"] // case["page_size"])) + case["spare"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)
    return {"select": _prepare_select, "reorder": _prepare_reorder, "fork": _prepare_fork, "compact": _prepare_compact,
            "copy": _prepare_copy}[case["op"]](case, gen)


def _prepare_select(case, gen):
    rows = case["requests"] * case["beams"]
    state = {"case": case, "logits": _cut(_logits(gen, rows, case["vocab"]), case)}
    score = -20.0 * torch.rand(case["requests"], 1, generator=gen, device="cuda")
    score = (score - 3.0 * torch.rand(case["requests"], case["beams"], generator=gen, device="cuda")).view(rows)
    order = _shuffled(gen, rows)
    ended, dead = case["ended"], case["dead"]
    token = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    token[order[:ended]] = case["vocab"] - 1 - case["vocab"] // 200
    score[order[ended:ended + dead]] = -INF
    state |= {"score": score, "ended": token, "norm": None}
    if case["norm"]:                    # by length; the beams that have ended are shorter
        length = torch.randint(20, 200, (case["requests"], 1), generator=gen, device="cuda").expand(-1, case["beams"])
        length = length.reshape(rows) - torch.where(token >= 0, 1 + order % 15, 0)
        state["norm"] = ((5.0 + length) / 6.0) ** 0.6
    return state


def _prepare_reorder(case, gen):
    rows, t, h, w = case["requests"] * case["beams"], case["tokens"], case["heads"], case["width"]
    shape = (h, t, w) if case["heads_first"] else (t, h, w)
    whole = _fill(gen, (case["buffers"], case["from_rows"], *shape), case["dtype"])
    state = {"case": case, "whole": whole, "states": list(whole.unbind(0)), "dim": 2 if case["heads_first"] else 1}
    if case["in_place"]:
        state["parent"] = _parents(gen, case["requests"], case["beams"], True)
        lengths = torch.tensor(_lengths(case, case["requests"], max(1, t // 4), t), device="cuda", dtype=torch.int32)
        state["length"] = lengths[_shuffled(gen, case["requests"])].repeat_interleave(case["beams"])
        return state
    state["parent"] = torch.randint(case["from_rows"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
    lengths = torch.tensor(_lengths(case, case["from_rows"], max(1, t // 4), t), device="cuda", dtype=torch.int32)
    state["length"] = lengths[_shuffled(gen, case["from_rows"])]
    state["to"] = torch.zeros((case["buffers"], rows, *shape), dtype=TYPES[case["dtype"]], device="cuda")
    state["out"] = list(state["to"].unbind(0))
    return state


def _prepare_fork(case, gen):
    requests, beams, ps = case["requests"], case["beams"], case["page_size"]
    rows, columns, pages = requests * beams, _columns(case), _pages(case)
    length = torch.tensor(_lengths(case, requests, case["shortest"], case["longest"]), device="cuda")
    length = length[_shuffled(gen, requests)]
    held, common = -(-length // ps), length // ps // 2
    # a request's pages one after the other: the common ones, then each beam's own
    own_pages = held - common
    start = torch.cumsum(common + beams * own_pages, 0) - (common + beams * own_pages)
    column = torch.arange(columns, device="cuda")
    beam = torch.arange(beams, device="cuda")[None, :, None]
    at = (start + common)[:, None, None] + beam * own_pages[:, None, None] + (column - common[:, None])[:, None, :]
    at = torch.where((column < common[:, None])[:, None, :], (start[:, None] + column)[:, None, :], at)
    at = torch.where((column < held[:, None])[:, None, :], at, -1).view(rows, columns)
    name = _shuffled(gen, pages)
    table = torch.where(at >= 0, name[at.clamp(min=0)], -1).int()
    refs = torch.bincount(table[table >= 0].long(), minlength=pages).int()
    parent = _parents(gen, requests, beams, False).view(requests, beams)
    order = _shuffled(gen, requests)
    kept, freed = order[:case["kept"]], order[case["kept"]:case["kept"] + case["freed"]]
    parent[kept] = torch.arange(rows, device="cuda", dtype=torch.int32).view(requests, beams)[kept]
    parent[freed] = -1
    pool = _fill(gen, (case["pools"], pages, ps * case["width"]), case["dtype"])
    return {"case": case, "pool": pool, "pools": list(pool.unbind(0)), "table": table, "refs": refs,
            "length": length.repeat_interleave(beams).int(), "parent": parent.view(-1)}


def _prepare_compact(case, gen):
    rows, columns, pages = case["rows"], case["columns"], case["pages"]
    live = _shuffled(gen, pages)[:case["live"]]
    # every live page in the table if it has room, some more than once; rows of every length
    count = torch.randint(columns + 1, (rows, 1), generator=gen, device="cuda")
    at = torch.randint(case["live"], (rows, columns), generator=gen, device="cuda")
    table = torch.where(torch.arange(columns, device="cuda") < count, live[at], -1).int()
    refs = torch.bincount(table[table >= 0].long(), minlength=pages).int()
    refs[live] += 1                     # what else holds a page: a pinned prefix, another unit
    pool = _fill(gen, (case["pools"], pages, case["page"]), case["dtype"])
    return {"case": case, "pool": pool, "pools": list(pool.unbind(0)), "table": table, "refs": refs,
            "keep": None if case["keep"] < 0 else case["keep"]}


def _prepare_copy(case, gen):
    pages, n = case["pages"], case["pairs"]
    order = _shuffled(gen, pages).int()
    pool = _fill(gen, (case["pools"], pages, case["page"]), case["dtype"])
    state = {"case": case, "pool": pool, "pools": list(pool.unbind(0)), "src": order[:n].contiguous(),
             "dst": order[pages - n:].contiguous(), "other": None, "to": None}
    if case["other"]:
        state["other"] = torch.zeros_like(pool)
        state["to"] = list(state["other"].unbind(0))
    return state


# ---- the operators, plain and own ------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"select": _own_select, "reorder": _own_reorder, "fork": _own_fork, "compact": _own_compact,
                "copy": _own_copy}[op](state)
    return {"select": _plain_select, "reorder": _plain_reorder, "fork": _plain_fork, "compact": _plain_compact,
            "copy": _plain_copy}[op](state)


def _own_select(s):
    from paper_2609_34645_b200 import logits
    case = s["case"]
    score, parent, token = logits.beam_select(s["logits"], s["score"], case["k"], beams=case["beams"], vocab=case["vocab"],
                                              ended=s["ended"], norm=s["norm"], settle=case["settle"])
    return {"score": score, "parent": parent, "token": token}


def _plain_select(s):
    case = s["case"]
    vocab, beams, k, requests = case["vocab"], case["beams"], case["k"], case["requests"]
    x = (s["logits"][0] if len(s["logits"]) == 1 else torch.cat(s["logits"], dim=1))[:, :vocab].float()
    # a whole number that orders as (larger value, lower token id) does
    bits = (x + 0.0).view(torch.int32).long()
    key = (torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF) << 32) - torch.arange(vocab, device=x.device)
    token = (-key.topk(min(k, vocab), dim=1).values) & 0xFFFFFFFF
    del key, bits
    top = x.amax(1, keepdim=True)
    # in 64 bits: what decides between hypotheses of different beams
    lse = top.double() + torch.log(torch.exp(x.double() - top).sum(1, keepdim=True))
    score = s["score"].double()[:, None]
    total = score - lse + x.gather(1, token)
    first = torch.arange(token.shape[1], device=x.device) == 0
    ended = s["ended"][:, None]
    total = torch.where(ended < 0, total, torch.where(first, score, -INF))
    token = torch.where(ended < 0, token, ended)
    rank = total if s["norm"] is None else total / s["norm"].double()[:, None]
    best = rank.view(requests, -1).argsort(dim=1, descending=True, stable=True)[:, :k]
    total, token = total.view(requests, -1).gather(1, best), token.view(requests, -1).gather(1, best)
    beam = best // min(k, vocab)
    none = total == -INF
    if case["settle"]:
        # a beam's best hypothesis stays in its row; the others take the rows that are left, in order
        place = torch.arange(k, device=x.device).expand(requests, k)
        mine = (beam[:, :, None] == torch.arange(beams, device=x.device)) & ~none[:, :, None]
        lead = torch.where(mine, place[:, :, None], k).amin(1)
        stays = (lead.gather(1, beam) == place) & ~none
        vacant = (lead < k).int().argsort(dim=1, stable=True)
        slot = torch.where(stays, beam, vacant.gather(1, (torch.cumsum(~stays, 1) - 1).clamp(min=0)))
        put = lambda v: torch.empty_like(v).scatter_(1, slot, v)                                    # noqa: E731
        total, token, beam, none = put(total), put(token), put(beam), put(none)
    parent = beam + beams * torch.arange(requests, device=x.device)[:, None]
    return {"score": total.float(), "parent": torch.where(none, -1, parent).int(), "token": torch.where(none, -1, token).int()}


def _own_reorder(s):
    from paper_2609_34645_b200 import cache
    if s["case"]["in_place"]:
        cache.reorder(s["states"], s["parent"], beams=s["case"]["beams"], length=s["length"], dim=s["dim"])
        return {"states": s["whole"]}
    cache.reorder(s["states"], s["parent"], length=s["length"], dim=s["dim"], out=s["out"])
    return {"states": s["to"]}


def _plain_reorder(s):
    to = s["whole"] if s["case"]["in_place"] else s["to"]
    parent, t = s["parent"].long(), s["case"]["tokens"]
    written = torch.arange(t, device=to.device) < s["length"][parent][:, None]
    written = written[:, None, :, None] if s["case"]["heads_first"] else written[:, :, None, None]
    to.copy_(torch.where(written, s["whole"][:, parent], to))
    return {"states": to}


def _own_fork(s):
    from paper_2609_34645_b200 import cache
    case = s["case"]
    table, length, refs, copies, status = cache.fork(s["pools"], s["table"], s["length"], s["refs"], s["parent"],
                                                     case["page_size"], room=case["room"])
    return {"table": table, "length": length, "refs": refs, "copies": copies, "status": status, "pool": s["pool"]}


def _plain_fork(s):
    case, table, refs, pool = s["case"], s["table"], s["refs"], s["pool"]
    ps, room = case["page_size"], case["room"]
    rows, columns = table.shape
    pages, dev = refs.shape[0], table.device
    parent = s["parent"].long()
    alive = (parent >= 0) & (parent < rows)
    parent = torch.where(alive, parent, 0)
    row, column = torch.arange(parent.shape[0], device=dev), torch.arange(columns, device=dev)
    kids = torch.zeros(rows, dtype=torch.int64, device=dev).scatter_add(0, parent, alive.long())
    lead = torch.full((rows,), parent.shape[0], device=dev).scatter_reduce(
        0, parent, torch.where(alive, row, parent.shape[0]), "amin")
    keeper = alive & (lead[parent] == row)
    length = s["length"].long().clamp(0, columns * ps)
    valid = (table >= 0) & (table < pages)
    # every row's pages lose the row and gain its children: full ones all of them, the others the first
    shared = column < (length // ps)[:, None]
    change = torch.where(shared, kids[:, None] - 1, torch.where(kids[:, None] > 0, 0, -1))
    at = torch.where(valid, table.long(), pages)
    refs1 = torch.nn.functional.pad(refs.long(), (0, 1)).scatter_add(0, at.view(-1), change.view(-1))[:pages]
    n = torch.where(alive, length[parent], 0)
    full, begun = (n // ps)[:, None], (n % ps > 0)[:, None]
    source, held = table[parent], valid[parent]
    new = torch.where(alive[:, None] & ((column < full) | keeper[:, None]), source, -1)
    until = torch.where(alive, -(-(n + room) // ps), 0)
    lacking = alive[:, None] & (column >= full) & (column < until[:, None]) & ~(keeper[:, None] & held)
    to_copy = (lacking & (column == full) & begun & held).any(1)
    # the j-th lacking page is the j-th free one
    free = refs1 <= 0
    missing = (lacking.sum() - free.sum()).clamp(min=0) + (until - columns).clamp(min=0).sum()
    fine = missing == 0
    rank = torch.cumsum(free, 0) - 1
    given = free & (rank < lacking.sum())
    by_rank = torch.full((pages + 1,), -1, device=dev).scatter(0, torch.where(given, rank, pages), torch.arange(pages, device=dev))
    j = torch.cumsum(lacking.view(-1), 0).view(lacking.shape) - 1
    new = torch.where(lacking, by_rank[j.clamp(0, pages - 1)], new.long())
    # copies, in the order of the rows
    to_copy = to_copy & fine
    first = full[:, 0].clamp(max=columns - 1)[:, None]
    pair = torch.cat([source.gather(1, first), new.gather(1, first)], 1)
    pair = torch.where(to_copy[:, None], pair, -1)[(~to_copy).int().argsort(stable=True)].int()
    src, dst = pair[to_copy.sum() > row].long().unbind(1)
    pool[:, dst] = pool[:, src]
    if_fine = lambda a, b: torch.where(fine, a, b) if a.shape == b.shape else a                     # noqa: E731
    left = torch.where(fine, free.sum() - lacking.sum(), (refs <= 0).sum())
    status = torch.stack([left, missing, to_copy.sum(), missing * 0]).int()
    return {"table": if_fine(new.int(), table), "length": if_fine(n.int(), s["length"]),
            "refs": if_fine(torch.where(given, 1, refs1).int(), refs), "copies": pair, "status": status, "pool": pool}


def _own_compact(s):
    from paper_2609_34645_b200 import cache
    table, refs, where, _, status = cache.compact(s["pools"], s["table"], s["refs"], keep=s["keep"])
    return {"table": table, "refs": refs, "map": where, "status": status, "pool": s["pool"]}


def _plain_compact(s):
    table, refs, pool = s["table"], s["refs"], s["pool"]
    pages, dev = refs.shape[0], refs.device
    page = torch.arange(pages, device=dev)
    live = refs > 0
    count = live.sum()
    keep = count if s["keep"] is None else torch.full_like(count, s["keep"])
    missing = (count - keep).clamp(min=0)
    goes = live & (page >= keep) & (missing == 0)
    moves = goes.sum()
    hole = ~live & (page < keep)
    src, dst = page[goes], page[hole & (torch.cumsum(hole, 0) <= moves)]
    where = torch.where(live, page, -1).scatter(0, src, dst)
    pool[:, dst] = pool[:, src]
    held = (table >= 0) & (table < pages)
    new = torch.where(held, where[table.clamp(0, pages - 1).long()], table)
    counts = torch.zeros_like(refs).scatter(0, torch.where(live, where, 0), torch.where(live, refs, 0), reduce="add")
    status = torch.stack([count, missing, moves, torch.where(missing > 0, pages, keep)])
    return {"table": new.int(), "refs": counts, "map": where.int(), "status": status.int(), "pool": pool}


def _own_copy(s):
    from paper_2609_34645_b200 import cache
    cache.copy(s["pools"], s["src"], s["dst"], to=s["to"])
    return {"pool": s["pool"] if s["other"] is None else s["other"]}


def _plain_copy(s):
    to = s["pool"] if s["other"] is None else s["other"]
    to[:, s["dst"].long()] = s["pool"][:, s["src"].long()]
    return {"pool": to}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    """A selection's scores: of every request all hypotheses, sorted.  What the other operators return is moved."""
    if case["op"] != "select":
        return None
    s = prepare(case, seed)
    beams, vocab, k, parts = case["beams"], case["vocab"], case["k"], []
    for g in range(case["requests"]):
        cut = slice(g * beams, (g + 1) * beams)
        x = torch.cat([p[cut] for p in s["logits"]], dim=1)[:, :vocab].double()
        score, ended = s["score"][cut].double(), s["ended"][cut].tolist()
        total = torch.log_softmax(x, 1) + score[:, None]
        for b, token in enumerate(ended):
            if token >= 0:
                total[b] = -INF
                total[b, token] = score[b]
        rank = total if s["norm"] is None else total / s["norm"][cut].double()[:, None]
        best = rank.view(-1).topk(k).indices
        value, beam = total.view(-1)[best], best // vocab
        if case["settle"]:
            row, left = torch.full((beams,), -1, device="cuda"), []
            for j, (v, b) in enumerate(zip(value.tolist(), beam.tolist())):
                if v > -INF and row[b] < 0:
                    row[b] = j
                else:
                    left.append(j)
            row[row < 0] = torch.tensor(left, device="cuda", dtype=torch.int64)
            value = value[row]
        parts.append(value)
    return {"score": torch.stack(parts), "parent": None, "token": None}
