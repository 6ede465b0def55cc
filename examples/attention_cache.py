"""The attention operators together, as a serving program and a training step
use them: prompts read with their key weights recorded, tokens decoded against
caches that are shortened to their heaviest rows when they are full, a batch
decoded over one common prefix, and the gradients of packed documents.

    python examples/attention_cache.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_16491_amd as F  # noqa: E402

HEADS, KV_HEADS, D = 8, 2, 64
SLOPES = [2.0 ** -(i + 1) for i in range(HEADS)]


def rows(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def decode(prompt=300, slots=320, steps=60, keep=256, recent=32, batch=2, seed=0):
    """Prompts of `prompt` tokens, then `steps` tokens each, in caches of `slots` rows that are cut to `keep` when full.
    Scores fall with the distance of the positions, which a cut leaves as they were.  Returns the last step's arguments
    and output."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    slopes = torch.tensor(SLOPES, device="cuda")
    k, v = (torch.zeros((batch, slots, KV_HEADS, D), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    k[:, :prompt], v[:, :prompt] = rows(g, batch, prompt, KV_HEADS, D), rows(g, batch, prompt, KV_HEADS, D)
    at = torch.zeros((batch, KV_HEADS, slots), device="cuda", dtype=torch.int32)
    at[:, :, :prompt] = torch.arange(prompt, device="cuda")
    weights = torch.zeros((batch, KV_HEADS, slots), device="cuda")
    # the prompt: token i sees 0 .. i
    place = torch.arange(prompt, device="cuda", dtype=torch.int32)
    causal = torch.stack([torch.zeros_like(place), place], -1)
    _, weights = F.attend(rows(g, batch, prompt, HEADS, D), k, v, causal, slopes=slopes, at_q=place.float().expand(batch, -1).contiguous(),
                          at_k=at.float(), weights=weights)
    used, lengths = prompt, torch.full((batch,), prompt, device="cuda", dtype=torch.int32)
    for step in range(steps):
        if used == slots:
            k2, v2, w2, at2, lengths = F.evict(k, v, weights, at, lengths, keep, recent=recent)
            for new, old in ((k2, k), (v2, v)):
                old[:, :keep] = new
            weights.zero_()
            weights[:, :, :keep], at[:, :, :keep] = w2, at2
            used = keep
        k[:, used], v[:, used] = rows(g, batch, KV_HEADS, D), rows(g, batch, KV_HEADS, D)
        at[:, :, used] = prompt + step
        weights[:, :, used] = 0.0
        used += 1
        lengths += 1
        q = rows(g, batch, 1, HEADS, D)
        args = dict(lr=torch.stack([torch.zeros_like(lengths), lengths - 1], -1).view(batch, 1, 2), slopes=slopes,
                    at_q=torch.full((batch, 1), float(prompt + step), device="cuda"), at_k=at.float())
        out, weights = F.attend(q, k, v, **args, weights=weights, weights_out=weights)
    return q, k, v, args, out, weights


def shared(batch=6, prefix=500, most=40, page=16, seed=1):
    """One token of each of `batch` requests over a common prefix and their own tails in pages."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-most // page)
    k_pages, v_pages = rows(g, batch * width, page, KV_HEADS, D), rows(g, batch * width, page, KV_HEADS, D)
    pages = torch.arange(batch * width, device="cuda", dtype=torch.int32).view(batch, width)
    lengths = (torch.arange(batch, device="cuda", dtype=torch.int32) * 7) % (most + 1)
    return F.attend_shared(rows(g, batch, HEADS, D), rows(g, prefix, KV_HEADS, D), rows(g, prefix, KV_HEADS, D), k_pages, v_pages, pages,
                           lengths, return_lse=True)


def train(sizes=(70, 130, 56), seed=2):
    """The gradients of one packed sequence of documents, scores capped."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(sizes)
    start = torch.cat([torch.full((n,), sum(sizes[:i]), dtype=torch.int32) for i, n in enumerate(sizes)]).cuda()
    lr = torch.stack([start, torch.arange(total, device="cuda", dtype=torch.int32)], -1).unsqueeze(0)
    q, k, v = (rows(g, 1, total, h, D).requires_grad_() for h in (HEADS, KV_HEADS, KV_HEADS))
    out = F.attend(q, k, v, lr, cap=30.0)
    out.float().square().sum().backward()
    return out.detach(), q.grad, k.grad, v.grad


if __name__ == "__main__":
    *_, args, out, weights = decode()
    print("decoded:", tuple(out.shape), "rows seen:", int(args["lr"][0, 0, 1]) + 1, "weight recorded:", float(weights.sum()))
    out, lse = shared()
    print("shared prefix:", tuple(out.shape), "log sums:", [round(x, 2) for x in lse[:, 0].tolist()])
    print("trained:", [tuple(t.shape) for t in train()])
