"""Cases for measuring the operators on an LM head's logits: ``process`` (a generation step: penalties for repeated
tokens, biases and grammar masks, with the greedy token and the log-sum-exp of the result), ``teacher_top`` (an
inference stage: a teacher's k largest logits and its log-sum-exp) and the distillation from them (a training
stage: ``forward``, ``backward`` and the two in one ``step``).

Logits are rows x vocabulary, cut into `tp` column shards as the head's rows are cut over tensor-parallel ranks,
each shard a tensor of its own; where the vocabulary does not divide, it is padded to a multiple of 128 * tp first
and the padding columns hold NaN, which nothing may read as a value.

`run` computes them with elementary torch operations in 32 bits (``own`` false) or through
``paper_2609_34645_b200.logits`` (``own`` true); `exact` gives the definition's values in 64 bits.
"""
import math

import torch

own = False

BF16, FP32 = "bf16", "fp32"
TYPES = {BF16: torch.bfloat16, FP32: torch.float32}
INF = math.inf


# ---- the cases -------------------------------------------------------------------------------------------------

def _process(name, rows, vocab, tp, dtype, out, history, bias, masked):
    return {"name": name, "op": "process", "rows": rows, "vocab": vocab, "tp": tp, "dtype": dtype, "out": out,
            "history": history, "bias": bias, "masked": masked}


def _top(name, rows, vocab, tp, dtype, k, temperature):
    return {"name": name, "op": "top", "rows": rows, "vocab": vocab, "tp": tp, "dtype": dtype, "k": k,
            "temperature": temperature}


def _distill(name, op, rows, vocab, tp, dtype, k, divergence, rest, temperature, skipped):
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "tp": tp, "dtype": dtype, "k": k,
            "divergence": divergence, "rest": rest, "temperature": temperature, "skipped": skipped}


def listed():
    return [
        # one request that decodes alone: the call's latency is all that counts
        _process("process 1 row", 1, 128256, 1, BF16, BF16, 300, 0, 0),
        # a decode step of 64 requests on the 8B model, head over 4 ranks, half of them under a grammar
        _process("process 64 rows tp4", 64, 128256, 4, BF16, FP32, 2000, 16, 32),
        # a large rollout batch on the 32B model's vocabulary with long histories, fp32 logits, all constrained
        _process("process 256 rows long", 256, 152064, 2, FP32, FP32, 16384, 0, 256),
        # an odd vocabulary, padded before the cut, many biases
        _process("process 37 rows odd", 37, 50257, 4, BF16, BF16, 777, 300, 19),
        # a teacher that scores a handful of positions
        _top("top 16 rows", 16, 128256, 1, BF16, 64, 1.0),
        # a teacher's batch of positions, head over 4 ranks
        _top("top 4096 rows tp4", 4096, 128256, 4, BF16, 64, 1.0),
        # fp32 logits of the 32B model's vocabulary, more entries kept
        _top("top 512 rows fp32", 512, 152064, 2, FP32, 128, 2.0),
        # odd rows, one after the other: no row but the first starts on a 16-byte boundary
        _top("top 333 rows odd", 333, 50257, 1, BF16, 20, 1.0),
        # the loss alone (a validation pass), Jensen-Shannon on fp32 logits
        _distill("forward 1024 rows fp32", "forward", 1024, 152064, 2, FP32, 128, "js", True, 1.0, 0),
        # the gradient from the forward's saved sums, teacher renormalised over its entries
        _distill("backward 2048 rows tp2", "backward", 2048, 128256, 2, BF16, 64, "forward_kl", False, 2.0, 0),
        # a training micro-batch of 8192 positions, a quarter of them prompt tokens that carry no loss
        _distill("step 8192 rows tp4", "step", 8192, 128256, 4, BF16, 64, "forward_kl", True, 1.0, 2048),
        # a small ragged batch on an odd vocabulary, the on-policy direction
        _distill("step 131 rows odd", "step", 131, 50257, 1, BF16, 32, "reverse_kl", True, 1.0, 40),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["process", "top", "forward", "backward", "step", "step"])
    vocab = rng.choice([128256, 152064, 50257, _spread(rng, 8000, 160000), _spread(rng, 8000, 160000) | 1])
    dtype = rng.choice([BF16, BF16, FP32])
    tp = rng.choice([1, 1, 2, 4, 8])
    rows = _spread(rng, 1, min(4096, 400_000_000 // vocab))
    if op == "process":
        rows = min(rows, 512)
        return {"op": op, "rows": rows, "vocab": vocab, "tp": tp, "dtype": dtype,
                "out": FP32 if dtype == FP32 else rng.choice([BF16, FP32]), "history": _spread(rng, 1, 16384),
                "bias": rng.choice([0, _spread(rng, 1, 300)]), "masked": rng.randint(0, rows)}
    k, temperature = _spread(rng, 1, 256), rng.choice([1.0, 1.0, 0.7, 2.0])
    if op == "top":
        return {"op": op, "rows": rows, "vocab": vocab, "tp": tp, "dtype": dtype, "k": k, "temperature": temperature}
    divergence = rng.choice(["forward_kl", "forward_kl", "reverse_kl", "js"])
    return {"op": op, "rows": rows, "vocab": vocab, "tp": tp, "dtype": dtype, "k": k, "divergence": divergence,
            "rest": divergence != "forward_kl" or rng.random() < 0.5, "temperature": temperature,
            "skipped": rng.choice([0, rng.randint(0, rows - 1)])}


def _size(dtype):
    return 2 if dtype == BF16 else 4


def work(case):
    r, v, es, op = case["rows"], case["vocab"], _size(case["dtype"]), case["op"]
    if op == "process":
        bytes_ = r * v * (es + _size(case["out"])) + r * (4 * case["history"] + 8 * case["bias"] + 8)
        bytes_ += case["masked"] * (v // 8)
        return {"bytes": bytes_, "flops": r * v * 8}
    if op == "top":
        return {"bytes": r * v * es + r * (8 * case["k"] + 4), "flops": r * v * 5}
    live = r - case["skipped"]
    entries = live * (8 * case["k"] + 8) + r * 8
    if op == "forward":
        return {"bytes": live * v * es + entries + r * 16, "flops": live * v * 4}
    if op == "backward":
        return {"bytes": (live + r) * v * es + entries + live * 16, "flops": live * v * 4}
    return {"bytes": (live + r) * v * es + entries, "flops": live * v * 8}


# ---- the inputs ------------------------------------------------------------------------------------------------

def _logits(gen, rows, vocab):
    """Rows as a language model gives them: a broad bulk, and a few dozen tokens that stand out of it."""
    x = torch.randn(rows, vocab, generator=gen, device="cuda").mul_(1.6)
    few = min(40, vocab)
    part = vocab // few
    at = torch.randint(part, (rows, few), generator=gen, device="cuda") + part * torch.arange(few, device="cuda")
    lift = torch.empty(rows, few, device="cuda").exponential_(0.35, generator=gen).add_(4.0)
    return x.scatter_(1, at, lift)


def _cut_width(case):
    v, tp = case["vocab"], case["tp"]
    if v % tp == 0:
        return v // tp
    return -(-v // (128 * tp)) * 128          # padded to a multiple of 128 * tp, then cut


def _cut(x, case, dtype):
    """The column shards, each a tensor of its own; padding columns are NaN."""
    w, v = _cut_width(case), case["vocab"]
    whole = torch.nn.functional.pad(x, (0, w * case["tp"] - v), value=math.nan)
    return [s.to(TYPES[dtype]).contiguous() for s in whole.split(w, dim=1)]


def _bits(allowed):
    """[rows, vocab] truth values as 32-bit words, token v in bit v % 32 of word v // 32."""
    rows, vocab = allowed.shape
    words = -(-vocab // 32)
    a = torch.nn.functional.pad(allowed, (0, words * 32 - vocab)).view(rows, words, 32).to(torch.int64)
    packed = (a << torch.arange(32, device=a.device)).sum(-1)
    return torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    rows, vocab = case["rows"], case["vocab"]
    rand = lambda *n: torch.rand(*n, generator=gen, device="cuda")                                  # noqa: E731
    x = _logits(gen, rows, vocab)
    state = {"case": case, "logits": _cut(x, case, case["dtype"])}
    if case["op"] == "process":
        length = case["history"]
        total = torch.full((rows,), length, device="cuda", dtype=torch.int32)
        total[1::2] = (rand(rows // 2) * length).int()                      # requests at every stage of their answer
        state["history"] = (rand(rows, length) ** 3 * vocab).int()          # few tokens often, many seldom
        state["total_len"] = total
        state["prompt_len"] = (rand(rows) * 0.5 * total).int()
        state["repetition"] = 1.0 + 0.3 * rand(rows)
        state["presence"] = rand(rows) - 0.2
        state["frequency"] = 0.5 * rand(rows)
        n = case["bias"]
        if n:
            part = vocab // n
            state["bias_ids"] = ((torch.arange(n, device="cuda") + rand(rows, n) * 0.999) * part).int()
            state["bias_values"] = torch.randn(rows, n, generator=gen, device="cuda") * 4
        m = case["masked"]
        if m:
            share = torch.where(rand(m, 1) < 0.5, 0.01, 0.9)                # grammars allow little, or nearly all
            allowed = rand(m, vocab) < share
            if m > 8:
                allowed[3] = False                                          # a grammar with no way on
            state["mask"] = _bits(allowed)
            which = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
            which[torch.randperm(rows, generator=gen, device="cuda")[:m]] = torch.arange(m, device="cuda").int()
            state["mask_row"] = which
        state["out"] = [torch.empty_like(s, dtype=TYPES[case["out"]]) for s in state["logits"]]
    elif case["op"] != "top":
        state |= _teacher(case, gen, x)
        if case["op"] == "backward":
            state["grad_loss"] = rand(rows) + 0.5
            state["saved"] = _saved(case, state)
        if case["op"] != "forward":
            state["grad"] = [torch.empty_like(s) for s in state["logits"]]
    return state


def _teacher(case, gen, x):
    """What an inference stage left behind: a teacher near the student, its k largest logits and log-sum-exp."""
    rows, vocab, k, t = case["rows"], case["vocab"], case["k"], case["temperature"]
    values, ids, lse = [], [], []
    for part in x.split(max(1, 200_000_000 // vocab)):
        y = part * 1.1 + 0.8 * torch.randn(part.shape, generator=gen, device="cuda")
        v, i = y.topk(k, dim=1)
        values.append(v)
        ids.append(i.int())
        lse.append(torch.logsumexp(y.double() / t, dim=1).float())
    weight = torch.rand(rows, generator=gen, device="cuda") + 0.5
    weight[torch.randperm(rows, generator=gen, device="cuda")[:case["skipped"]]] = 0.0
    return {"values": torch.cat(values), "ids": torch.cat(ids), "weight": weight,
            "lse": torch.cat(lse) if case["rest"] else None}


def _saved(case, state):
    """A forward pass's saved sums: the row's largest logit, the sums of exp((x - max) / T) over all tokens and over
    those the teacher's entries leave, and the divergence."""
    saved = []
    for a in range(0, case["rows"], 256):
        b = min(case["rows"], a + 256)
        x = _whole([s[a:b] for s in state["logits"]], case["vocab"]).double()
        lse = None if state["lse"] is None else state["lse"][a:b].double()
        saved.append(_definition(case, x, state["ids"][a:b].long(), state["values"][a:b].double(), lse)[2])
    return torch.cat(saved).float()


# ---- the operators, plain and own ------------------------------------------------------------------------------

def _whole(shards, vocab):
    return (shards[0] if len(shards) == 1 else torch.cat(shards, dim=1))[:, :vocab]


def _split(x, state):
    """The valid columns of every shard."""
    return list(x.split(_cut_width(state["case"]), dim=1))


def _valid(shards, case):
    w, v = _cut_width(case), case["vocab"]
    return [s[:, :min(w, v - i * w)] for i, s in enumerate(shards) if i * w < v]


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_process(state) if op == "process" else _own_top(state) if op == "top" else _own_distill(state)
    return _plain_process(state) if op == "process" else _plain_top(state) if op == "top" else _plain_distill(state)


def _own_process(s):
    from paper_2609_34645_b200 import logits
    out, token, lse = logits.process(
        s["logits"], vocab=s["case"]["vocab"], out=s["out"], history=s["history"], prompt_len=s["prompt_len"],
        total_len=s["total_len"], repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
        bias_ids=s.get("bias_ids"), bias_values=s.get("bias_values"), mask=s.get("mask"), mask_row=s.get("mask_row"))
    return {"out": _valid(out, s["case"]), "token": token, "lse": lse}


def _plain_process(s):
    case = s["case"]
    vocab = case["vocab"]
    x = _whole(s["logits"], vocab).float()
    place = torch.arange(s["history"].shape[1], device=x.device)
    ids = torch.where(place < s["total_len"][:, None], s["history"], vocab).long()
    answered = torch.where(place >= s["prompt_len"][:, None], ids, vocab)
    blank = torch.zeros(x.shape[0], vocab + 1, device=x.device)
    seen = blank.scatter(1, ids, 1.0)[:, :vocab] > 0
    count = blank.scatter_add(1, answered, torch.ones_like(answered, dtype=torch.float32))[:, :vocab]
    rho = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
    x = x - s["frequency"][:, None] * count
    x = x - s["presence"][:, None] * (count > 0)
    if "bias_ids" in s:
        x = x + blank.scatter(1, s["bias_ids"].long(), s["bias_values"])[:, :vocab]
    if "mask" in s:
        token = torch.arange(vocab, device=x.device)
        words = s["mask"][s["mask_row"].clamp(min=0).long()][:, token >> 5]
        allowed = ((words >> (token & 31)) & 1) > 0
        x = torch.where(allowed | (s["mask_row"] < 0)[:, None], x, -INF)
    out = x.to(TYPES[case["out"]])
    x = out.float()
    top = x.amax(1, keepdim=True)
    at = torch.where((x == top) & (x > -INF), torch.arange(vocab, device=x.device), vocab).amin(1)
    base = torch.where(top > -INF, top, 0.0)
    lse = base[:, 0] + torch.log(torch.exp(x - base).sum(1))
    return {"out": _split(out, s), "token": torch.where(at < vocab, at, -1).int(), "lse": lse}


def _own_top(s):
    from paper_2609_34645_b200 import logits
    case = s["case"]
    values, ids, lse = logits.teacher_top(s["logits"], case["k"], vocab=case["vocab"], temperature=case["temperature"])
    return {"values": values, "ids": ids, "lse": lse}


def _plain_top(s):
    case = s["case"]
    x = _whole(s["logits"], case["vocab"]).float()
    # a whole number that orders as (larger value, lower token id) does
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF)
    key = (order << 32) - torch.arange(case["vocab"], device=x.device)
    best = key.topk(case["k"], dim=1).values
    ids = (-best) & 0xFFFFFFFF
    z = x / case["temperature"]
    top = z.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    return {"values": x.gather(1, ids), "ids": ids.int(), "lse": lse}


def _own_distill(s):
    from paper_2609_34645_b200 import logits
    case = s["case"]
    how = {"vocab": case["vocab"], "lse": s["lse"], "weight": s["weight"], "divergence": case["divergence"],
           "temperature": case["temperature"]}
    if case["op"] == "forward":
        loss, saved = logits.distill_forward(s["logits"], s["ids"], s["values"], **how)
        return {"loss": loss, "saved": saved}
    if case["op"] == "backward":
        grad = logits.distill_backward(s["logits"], s["ids"], s["values"], s["saved"], grad_loss=s["grad_loss"],
                                       grad=s["grad"], **how)
        return {"grad": _valid(grad, case)}
    loss, grad = logits.distill_step(s["logits"], s["ids"], s["values"], grad=s["grad"], **how)
    return {"loss": loss, "grad": _valid(grad, case)}


def _plain_distill(s):
    case = s["case"]
    vocab, t = case["vocab"], case["temperature"]
    live = s["weight"] != 0
    x = _whole(s["logits"], vocab).float()
    ids = s["ids"].long()
    x_top = x.gather(1, ids)
    # the student: entries and rest, from the sums
    if case["op"] == "backward":
        m, total, rest, divergence = s["saved"][:, 0:1], s["saved"][:, 1:2], s["saved"][:, 2:3], s["saved"][:, 3:4]
    else:
        m = x.amax(1, keepdim=True)
        rest = torch.exp((x.scatter(1, ids, -INF) - m) / t).sum(1, keepdim=True)
        total = rest + torch.exp((x_top - m) / t).sum(1, keepdim=True)
    log_q = torch.cat([(x_top - m) / t, torch.log(rest)], 1) - torch.log(total)
    # the teacher: entries, and what they leave
    y = s["values"] / t
    if s["lse"] is None:
        top = y.amax(1, keepdim=True)
        p = torch.exp(y - top)
        p = torch.cat([p / p.sum(1, keepdim=True), torch.zeros_like(m)], 1)
    else:
        p = torch.exp(y - s["lse"][:, None])
        p = torch.cat([p, (1 - p.sum(1, keepdim=True)).clamp(min=0)], 1)
    q = torch.exp(log_q)
    if case["divergence"] == "forward_kl":
        term = torch.where(p > 0, p * (torch.log(p) - log_q), 0.0)
        slope = torch.where(p > 0, -p / q, 0.0)
        mean = -p.sum(1, keepdim=True)
    elif case["divergence"] == "reverse_kl":
        p = torch.cat([p[:, :-1], p[:, -1:].clamp(min=2.0 ** -24)], 1)
        slope = log_q - torch.log(p)
        term = q * slope
        mean = None
    else:
        mix = 0.5 * p + 0.5 * q
        slope = 0.5 * (log_q - torch.log(mix))
        term = torch.where(p > 0, 0.5 * p * (torch.log(p) - torch.log(mix)), 0.0) + q * slope
        mean = (q * slope).sum(1, keepdim=True)
    if case["op"] != "backward":
        divergence = term.sum(1, keepdim=True)
    loss = torch.where(live, divergence[:, 0] * s["weight"], 0.0)
    if case["op"] == "forward":
        saved = torch.cat([m, total, rest, divergence], 1)
        return {"loss": loss, "saved": torch.where(live[:, None], saved, 0.0)}
    scale = s["weight"][:, None] * (s["grad_loss"][:, None] if case["op"] == "backward" else 1.0) / t
    slope = slope - (divergence if mean is None else mean)
    grad = torch.exp((x - m) / t) * (slope[:, -1:] * scale / total)
    grad = grad.scatter(1, ids, q[:, :-1] * slope[:, :-1] * scale)
    grad = torch.where(live[:, None], grad, 0.0).to(TYPES[case["dtype"]])
    if case["op"] == "backward":
        return {"grad": _split(grad, s)}
    return {"loss": loss, "grad": _split(grad, s)}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _definition(case, x, ids, values, lse):
    """(divergence, d divergence / d logits, saved sums) of some rows, by the groups' probabilities: every token of
    the teacher's entries is a group of its own, all other tokens are one."""
    t, k = case["temperature"], case["k"]
    rows, vocab = x.shape
    z = x / t
    logq_all = torch.log_softmax(z, 1)
    group = torch.full((rows, vocab), k, device=x.device)
    group.scatter_(1, ids, torch.arange(k, device=x.device).expand(rows, k))
    q = torch.zeros(rows, k + 1, dtype=torch.float64, device=x.device).scatter_add_(1, group, logq_all.exp())
    if lse is None:
        p = torch.softmax(values / t, 1)
        p = torch.cat([p, torch.zeros(rows, 1, dtype=torch.float64, device=x.device)], 1)
    else:
        p = torch.exp(values / t - lse[:, None])
        p = torch.cat([p, (1 - p.sum(1, keepdim=True)).clamp(min=0)], 1)
    if case["divergence"] == "forward_kl":
        d = torch.special.xlogy(p, p / q).sum(1)
        f = -p / q
    elif case["divergence"] == "reverse_kl":
        p[:, k] = p[:, k].clamp(min=2.0 ** -24)
        f = torch.log(q / p)
        d = (q * f).sum(1)
    else:
        mix = (p + q) / 2
        f = torch.log(q / mix) / 2
        d = (torch.special.xlogy(p, p / mix) + torch.special.xlogy(q, q / mix)).sum(1) / 2
    grad = logq_all.exp() * (f - (q * f).sum(1, keepdim=True)).gather(1, group) / t
    m = x.amax(1)
    total = torch.exp(torch.logsumexp(z, 1) - m / t)
    return d, grad, torch.stack([m, total, total * q[:, k], d], 1)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "process":
        return _exact_process(state)
    if case["op"] == "top":
        return _exact_top(state)
    vocab, parts = case["vocab"], []
    for a in range(0, case["rows"], 256):
        cut = slice(a, a + 256)
        x = _whole([s[cut] for s in state["logits"]], vocab).double()
        lse = None if state["lse"] is None else state["lse"][cut].double()
        d, grad, saved = _definition(case, x, state["ids"][cut].long(), state["values"][cut].double(), lse)
        weight = state["weight"][cut].double()
        scale = weight * (state["grad_loss"][cut].double() if case["op"] == "backward" else 1.0)
        out = {"loss": d * weight}
        if case["op"] == "forward":
            out["saved"] = saved * (weight != 0)[:, None]
        else:
            out["grad"] = grad * scale[:, None]
        parts.append(out)
    whole = {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    if "grad" in whole:
        whole["grad"] = list(whole["grad"].split(_cut_width(case), dim=1))
    if case["op"] == "backward":
        del whole["loss"]
    return whole


def _exact_process(s):
    case = s["case"]
    rows, vocab = case["rows"], case["vocab"]
    x = _whole(s["logits"], vocab).double()
    place = torch.arange(case["history"], device="cuda")
    flat = s["history"].long() + torch.arange(rows, device="cuda")[:, None] * vocab
    inside = place < s["total_len"][:, None]
    answer = inside & (place >= s["prompt_len"][:, None])
    seen = torch.bincount(flat[inside], minlength=rows * vocab).view(rows, vocab) > 0
    count = torch.bincount(flat[answer], minlength=rows * vocab).view(rows, vocab)
    rho = s["repetition"].double()[:, None].expand(rows, vocab)
    x[seen & (x > 0)] /= rho[seen & (x > 0)]
    low = seen & (x < 0)
    x[low] *= rho[low]
    x -= s["frequency"].double()[:, None] * count + s["presence"].double()[:, None] * (count > 0)
    if "bias_ids" in s:
        row = torch.arange(rows, device="cuda")[:, None].expand(rows, case["bias"])
        x[row, s["bias_ids"].long()] += s["bias_values"].double()
    if "mask" in s:
        bit = torch.arange(32, device="cuda")
        allowed = ((s["mask"].long()[:, :, None] >> bit) & 1).view(case["masked"], -1)[:, :vocab] == 1
        under = s["mask_row"] >= 0
        banned = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda")
        banned[under] = ~allowed[s["mask_row"][under].long()]
        x.masked_fill_(banned, -INF)
    return {"out": list(x.split(_cut_width(case), dim=1)), "token": None, "lse": torch.logsumexp(x, 1)}


def _exact_top(s):
    case = s["case"]
    values, lse = [], []
    for a in range(0, case["rows"], 512):
        x = _whole([p[a:a + 512] for p in s["logits"]], case["vocab"]).double()
        values.append(x.sort(dim=1, descending=True).values[:, :case["k"]].clone())
        lse.append(torch.logsumexp(x / case["temperature"], 1))
    return {"values": torch.cat(values), "ids": None, "lse": torch.cat(lse)}
