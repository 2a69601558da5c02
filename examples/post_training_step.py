"""A post-training loop in small, with the steps of its three model-stages on the LM head's logits:

  generation   the actor's weights come from the training layout by a transition (TP2, padded vocabulary -> TP4, padded
               vocabulary); each decode step penalises repeated tokens, keeps to a grammar and takes the greedy token
  inference    a teacher scores the same positions and leaves its top logits
  training     the actor is distilled from them under the training layout, and its head is updated

The decoder below the head is left out: hidden states are a fixed projection of the token before.  Run on a B200:

  python examples/post_training_step.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_34645_b200 import binding as B                      # noqa: E402
from paper_2609_34645_b200 import logits as L                       # noqa: E402

LAYERS, HIDDEN, HEADS, KV_HEADS, FFN, VOCAB = 2, 256, 8, 4, 512, 1000
ROWS, PROMPT, ANSWER, TOP = 16, 6, 10, 32
TRAIN = B.Plan(2, 1, 0, B.VOCAB_PADDED)
GENERATE = B.Plan(4, 1, 0, B.VOCAB_PADDED)


def head_shards(desc, plan, bufs):
    """The LM head's [V_pad / tp, H] block in each shard buffer, as views."""
    head = desc.num_tensors() - 1
    views = []
    for s, buf in enumerate(bufs):
        off, rows, cols, _ = desc.tensor_slice(plan, s, head)
        if rows:
            views.append(buf[off:off + rows * cols * 2].view(torch.bfloat16).view(rows, cols))
    return views


def main(steps=6, device="cuda"):
    gen = torch.Generator(device).manual_seed(0)
    desc = B.ModelDesc(LAYERS, HIDDEN, HEADS, KV_HEADS, FFN, VOCAB, B.BF16)
    sync = desc.compile(TRAIN, GENERATE)                            # the weight sync, actor-training -> actor-generation
    sync.prepare()
    train = [(torch.randn(n // 2, generator=gen, device=device) * 0.05).bfloat16().view(torch.uint8) for n in desc.shard_sizes(TRAIN)]
    generate = [torch.zeros(n, dtype=torch.uint8, device=device) for n in desc.shard_sizes(GENERATE)]
    head, actor = head_shards(desc, TRAIN, train), head_shards(desc, GENERATE, generate)
    teacher = torch.randn(VOCAB, HIDDEN, generator=gen, device=device).mul_(0.2).bfloat16()
    embed = torch.randn(VOCAB, HIDDEN, generator=gen, device=device).bfloat16()
    stream = torch.cuda.current_stream().cuda_stream
    # a grammar that forbids every third token
    allowed = torch.arange(-(-VOCAB // 32) * 32, device=device).view(-1, 32) % 3 > 0
    words = (allowed.long() << torch.arange(32, device=device)).sum(1)
    mask = torch.where(words >= 1 << 31, words - (1 << 32), words).int().view(1, -1)
    which = torch.where(torch.arange(ROWS, device=device) % 2 == 0, 0, -1).int()     # half of the requests are under it
    rho = torch.full((ROWS,), 1.2, device=device)
    presence = torch.full((ROWS,), 0.3, device=device)
    prompt_len = torch.full((ROWS,), PROMPT, device=device, dtype=torch.int32)
    losses = []
    for step in range(steps):
        sync.run([b.data_ptr() for b in train], [b.data_ptr() for b in generate], stream)

        # generation: one token of every request at a time
        history = torch.zeros(ROWS, PROMPT + ANSWER, dtype=torch.int32, device=device)
        history[:, :PROMPT] = torch.randint(VOCAB, (ROWS, PROMPT), generator=gen, device=device)
        for n in range(PROMPT, PROMPT + ANSWER):
            h = embed[history[:, n - 1].long()]
            logits = [h @ w.T for w in actor]
            total = torch.full((ROWS,), n, device=device, dtype=torch.int32)
            _, token, _ = L.process(logits, vocab=VOCAB, out=logits, history=history, prompt_len=prompt_len, total_len=total,
                                    repetition=rho, presence=presence, mask=mask, mask_row=which)
            history[:, n] = token

        # inference: the teacher on the positions that led to the answers
        h = embed[history[:, PROMPT - 1:-1].reshape(-1).long()]
        values, ids, lse = L.teacher_top(h @ teacher.T, TOP)

        # training: the loss and the gradient of the actor's logits in its training layout, and a step of its head
        logits = [h @ w.T for w in head]
        loss, grad = L.distill_step(logits, ids, values, vocab=VOCAB, lse=lse, divergence="forward_kl",
                                    grad=[torch.zeros_like(x) for x in logits])
        for w, g in zip(head, grad):
            w -= (1.0 / h.shape[0] * (g.float().T @ h.float())).bfloat16()
        after, _ = L.distill_forward([h @ w.T for w in head], ids, values, vocab=VOCAB, lse=lse, divergence="forward_kl")
        losses.append(torch.stack([loss.mean(), after.mean()]))
    return torch.stack(losses).tolist(), history, mask, which


if __name__ == "__main__":
    for step, (before, after) in enumerate(main()[0]):
        print(f"step {step}: distillation loss {before:.4f}, after the update {after:.4f}")
