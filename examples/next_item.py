#!/usr/bin/env python3
"""A causal next-item model on the operators of this library: trained on whole histories, then served one item at a time from
the states it keeps.

    python examples/next_item.py [--steps 60] [--items 500] [--dtype bf16] [--mixer delta|decay] [--dropout 0.1] [--slates 4]

Synthetic histories: every user walks through the catalogue with a stride of their own, so the next item follows from the
history and from nothing else.  One layer: E = sqrt(D) * W[id] + P; q, k, v, decay and beta are projections of it; the
delta rule mixes the history; scores are products with the item table.  Served scores are compared with those of the
whole history in one call.

With `--mixer decay` the history is mixed by linear attention with a learned decay for each head, E and what is added to it are
dropped in part while it is trained, and the layer ends in a seam: X = E + gate * drop(norm(O)), scores from norm(X).  `--slates K`
then continues every history by the best K slates of three items, by beam search: the states follow their beams.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_06935_amd import binding                                               # noqa: E402
from paper_2602_06935_amd.autograd import (decay_attention, dropout, gated_delta_attention, item_embedding,   # noqa: E402
                                           residual_norm)


class NextItem(torch.nn.Module):
    def __init__(self, items, longest, width=64, heads=2, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.head_dim, self.scale = heads, width // heads, math.sqrt(width)
        normal = lambda *s: torch.nn.Parameter((torch.randn(*s) * 0.1).to(dtype))        # noqa: E731
        self.W, self.P = normal(items, width), normal(longest, width)                   # item 0 is the padding
        self.qkv = torch.nn.Linear(width, 3 * width, dtype=dtype)
        self.gates = torch.nn.Linear(width, 2 * heads, dtype=dtype)
        self.out = torch.nn.Linear(width, width, dtype=dtype)

    def heads_of(self, E):
        B, N, _ = E.shape
        q, k, v = (t.reshape(B, N, self.heads, self.head_dim).contiguous() for t in self.qkv(E).chunk(3, -1))
        g, beta = self.gates(E).float().chunk(2, -1)
        return q, k, v, -torch.nn.functional.softplus(g - 3.0).contiguous(), torch.sigmoid(beta).contiguous()

    def scores(self, E, O):
        h = E + self.out(O.flatten(2))
        return h.float() @ self.W.float().t() / self.scale

    def forward(self, ids):
        """Scores of the next item after every position of [B,N] histories, padded with 0 on the left."""
        E = item_embedding(ids, self.W, self.P, scale=self.scale, padding_idx=0)
        mask = (ids != 0).to(torch.uint8)
        O = gated_delta_attention(*self.heads_of(E), mask, layout="bnhd")
        return self.scores(E, O)

    @torch.no_grad()
    def take_in(self, ids, state, position):
        """One more item for every user: scores of the next, the states replaced in place."""
        E = binding.cotten_embed_fwd(ids, self.W, self.P, scale=self.scale, padding_idx=0, position_offset=position)
        q, k, v, g, beta = self.heads_of(E)
        mask = (ids != 0).to(torch.uint8)
        O = binding.cotten_delta_fwd(q, k, v, g, beta, mask, layout="bnhd", initial_state=state, final_state=state)
        return self.scores(E, O)[:, 0]


class DecayItem(torch.nn.Module):
    """The same with a decay for each head, dropout and a seam behind the attention.  `p` drops while the model trains; every
    call draws anew."""
    def __init__(self, items, longest, width=64, heads=2, dtype=torch.bfloat16, p=0.0):
        super().__init__()
        self.heads, self.head_dim, self.scale, self.p = heads, width // heads, math.sqrt(width), p
        normal = lambda *s: torch.nn.Parameter((torch.randn(*s) * 0.1).to(dtype))        # noqa: E731
        self.W, self.P = normal(items, width), normal(longest, width)                   # item 0 is the padding
        self.qkv = torch.nn.Linear(width, 3 * width, dtype=dtype)
        self.out = torch.nn.Linear(width, width, dtype=dtype)
        self.forget = torch.nn.Parameter(torch.linspace(0.0, -4.0, heads))              # from half of a state a token to little
        ones = lambda: torch.nn.Parameter(torch.ones(width, dtype=dtype))                # noqa: E731
        self.after, self.gate, self.before = ones(), ones(), ones()
        self.seed, self.calls = 0, 0

    def heads_of(self, E):
        B, N, _ = E.shape
        return (t.reshape(B, N, self.heads, self.head_dim).contiguous() for t in self.qkv(E).chunk(3, -1))

    def rates(self):
        return -torch.nn.functional.softplus(self.forget.float())

    def seam(self):
        return dict(post_weight=self.after, gate=self.gate, next_weight=self.before)

    def scores(self, H):
        return H.float() @ self.W.float().t() / self.scale

    def forward(self, ids):
        """Scores of the next item after every position of [B,N] histories, padded with 0 on the left."""
        p = self.p if self.training else 0.0
        E = item_embedding(ids, self.W, self.P, scale=self.scale, padding_idx=0)
        if p > 0:
            E = dropout(E, p, seed=self.seed, offset=2 * self.calls)
        O = decay_attention(*self.heads_of(E), self.rates(), (ids != 0).to(torch.uint8), layout="bnhd")
        _, H = residual_norm(E, self.out(O.flatten(2)), p=p, seed=self.seed, offset=2 * self.calls + 1, **self.seam())
        self.calls += 1
        return self.scores(H)

    @torch.no_grad()
    def take_in(self, ids, state, position):
        """One more item for every user: scores of the next, the states replaced in place."""
        E = binding.cotten_embed_fwd(ids, self.W, self.P, scale=self.scale, padding_idx=0, position_offset=position)
        O = binding.cotten_decay_fwd(*self.heads_of(E), self.rates(), (ids != 0).to(torch.uint8), layout="bnhd",
                                     initial_state=state, final_state=state)
        _, H = binding.cotten_residual_fwd(E, self.out(O.flatten(2)), **self.seam())
        return self.scores(H)[:, 0]


@torch.no_grad()
def slates(model, state, scores, position, beams, length):
    """The `beams` best continuations of every history by `length` items, from its state and the scores of the next item:
    (items [B,beams,length], their log-probabilities [B,beams])."""
    B, V = scores.shape
    state = state[:, None].repeat(1, beams, 1, 1, 1)
    total = torch.full((B, beams), float("-inf"), device=scores.device)
    total[:, 0] = 0.0                                             # (all beams are one still)
    items = torch.zeros(B, beams, length, dtype=torch.int32, device=scores.device)
    logits = scores[:, None].repeat(1, beams, 1)
    for t in range(length):
        logits[..., 0] = float("-inf")                            # the padding is no item
        total, parents, tokens = binding.cotten_beam_select(logits.contiguous(), total)
        binding.cotten_beam_reorder(items, parents)
        items[:, :, t] = tokens
        if t + 1 < length:
            binding.cotten_beam_reorder(state, parents)
            logits = model.take_in(tokens.reshape(-1, 1), state.flatten(0, 1), position + t).reshape(B, beams, V)
    return items, total


def histories(users, length, items, gen):
    stride = torch.randint(1, 8, (users, 1), generator=gen)
    start = torch.randint(0, items, (users, 1), generator=gen)
    ids = (start + stride * torch.arange(length)[None, :]) % (items - 1) + 1
    short = torch.randint(0, length // 2, (users, 1), generator=gen)
    return torch.where(torch.arange(length)[None, :] < short, 0, ids)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--items", type=int, default=500)
    ap.add_argument("--users", type=int, default=256)
    ap.add_argument("--length", type=int, default=50)
    ap.add_argument("--dtype", choices=("f32", "bf16", "f16"), default="bf16")
    ap.add_argument("--mixer", choices=("delta", "decay"), default="delta")
    ap.add_argument("--dropout", type=float, default=0.0, help="with --mixer decay")
    ap.add_argument("--slates", type=int, default=0, help="beams of a search over three more items")
    args = ap.parse_args()
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[args.dtype]
    torch.manual_seed(0)
    gen = torch.Generator().manual_seed(0)
    longest = args.length + (3 if args.slates else 0)
    if args.mixer == "delta":
        model = NextItem(args.items, longest, dtype=dtype).cuda()
    else:
        model = DecayItem(args.items, longest, dtype=dtype, p=args.dropout).cuda()
    master = [p.detach().float().clone().requires_grad_() for p in model.parameters()]    # the optimizer's, in 32 bits
    optimizer = torch.optim.Adam(master, lr=1e-2)
    losses = []
    for step in range(args.steps):
        ids = histories(args.users, args.length, args.items, gen).cuda()
        scores = model(ids[:, :-1].contiguous())
        target = torch.where(ids[:, :-1] != 0, ids[:, 1:], -100)
        loss = torch.nn.functional.cross_entropy(scores.flatten(0, 1), target.flatten(), ignore_index=-100)
        loss.backward()
        for p, m in zip(model.parameters(), master):
            m.grad, p.grad = p.grad.float(), None
        optimizer.step()
        with torch.no_grad():
            for p, m in zip(model.parameters(), master):
                p.copy_(m)
        losses.append(loss.item())
        if step % 10 == 0 or step == args.steps - 1:
            print(f"step {step}: loss {losses[-1]:.3f}", flush=True)

    model.eval()
    ids = histories(args.users, args.length, args.items, gen).cuda()
    with torch.no_grad():
        whole = model(ids)
    state = torch.zeros(args.users, model.heads, model.head_dim, model.head_dim, device="cuda")
    far = 0.0
    for t in range(args.length):
        served = model.take_in(ids[:, t:t + 1].contiguous(), state, t)
        far = max(far, ((served - whole[:, t]).norm() / whole[:, t].norm()).item())
    print(f"served item by item against the whole history: {far:.1e}")
    if args.slates:
        items, total = slates(model, state, served.clone(), args.length, args.slates, 3)
        stride = (ids[:, -1] - ids[:, -2]) % (args.items - 1)
        right = (ids[:, -1:].long() - 1 + stride[:, None] * torch.arange(1, 4, device="cuda")) % (args.items - 1) + 1
        found = (items == right[:, None]).all(-1).any(1).float().mean().item()
        print(f"the walk's next three items are among {args.slates} slates of {found:.0%} of the users")
    return losses, far


if __name__ == "__main__":
    main()
