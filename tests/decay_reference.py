"""The decay attention from its definition, token by token in 64 bits on the CPU, with gradients by differentiating that; inputs
for the tests.

Bounds: those of the gated delta rule (`delta_reference.check`), by the same count.  Nothing is rounded below 24 significant bits
before a result is stored, so a fp32 result carries the fp32 rounding errors of the sums of d + 32 products that make it and of the
chunks before it, which add up as far as the decay lets them: below 1e-5.  A 16-bit result is off by its own rounding besides.  A
gradient of the decays is a sum over tokens of either sign of such terms, each times its distance: 1e-5 of the root of the sum of their
squares."""
import math

import torch

from delta_reference import DTYPES, FP32_BAR, check  # noqa: F401


def inputs(B, H, N, d, dtype, seed=0, mask=None, states=False, rates=(1e-3, 1.0)):
    """CPU tensors in [B,H,N,...] order, floats rounded to `dtype` where the operator takes that type."""
    gen = torch.Generator().manual_seed(seed)
    x = {n: torch.randn(B, H, N, d, generator=gen).to(dtype) for n in ("q", "k", "v", "dO")}
    low, high = math.log(rates[0]), math.log(rates[1])
    x["g"] = -torch.exp(low + (high - low) * torch.rand(H, generator=gen))
    x["mask"] = None
    if mask is not None:
        lengths = torch.randint(1, N + 1, (B,), generator=gen)
        m = torch.arange(N)[None, :] >= (N - lengths)[:, None]            # histories padded on the left
        if mask == "right":
            m = m.flip(1)
        if mask == "holes":
            m = torch.rand(B, N, generator=gen) < 0.6
        if mask in ("holes", "empty"):
            m[-1] = False                                                 # a sequence without any valid token
        x["mask"] = m.to(torch.uint8)
    x["S0"] = torch.randn(B, H, d, d, generator=gen) * 0.3 if states else None
    x["dS1"] = torch.randn(B, H, d, d, generator=gen) * 0.3 if states else None
    return x


def reference(x, scale=1.0, eps=1e-6, grads=True):
    """O, S1 and, with `grads`, dQ, dK, dV, dg, dS0 (all [B,H,N,...], float64); "dg_size": the root of the sum of the squares of the
    terms of dg."""
    q, k, v, g = (x[n].detach().double() for n in ("q", "k", "v", "g"))
    B, H, N, d = q.shape
    live = torch.ones(B, N, dtype=torch.bool) if x["mask"] is None else x["mask"] != 0
    k, v = (torch.where(live[:, None, :, None], t, 0.0) for t in (k, v))    # what masked rows hold is never looked at
    S0 = torch.zeros(B, H, d, d, dtype=torch.float64) if x["S0"] is None else x["S0"].double()
    rates = g[None, :, None].expand(B, H, N).contiguous()                   # (a leaf per token: their gradients are the terms of dg)
    leaves = [t.requires_grad_(grads) for t in (q, k, v, rates, S0)]
    with torch.set_grad_enabled(grads):
        qn, kn = (t / (t.square().sum(-1, keepdim=True) + eps).sqrt() for t in (q, k))
        S, o = S0, []
        for t in range(N):
            on = live[:, None, t, None, None]
            S = torch.where(on, rates[:, :, t, None, None].exp() * S + kn[:, :, t, :, None] * v[:, :, t, None, :], S)
            o.append((qn[:, :, t, :, None] * S).sum(-2))
        O = scale * torch.stack(o, 2)
    out = {"O": O.detach(), "S1": S.detach()}
    if grads:
        outputs, up = [O], [x["dO"].double()]
        if x["dS1"] is not None:
            outputs, up = [O, S], up + [x["dS1"].double()]
        dq, dk, dv, terms, dS0 = torch.autograd.grad(outputs, leaves, up, allow_unused=True)
        out.update(dQ=dq, dK=dk, dV=dv, dg=terms.sum((0, 2)), dS0=dS0, dg_size=terms.square().sum().sqrt().item())
    return out


def check_decays(got, ref):
    """The whole gradient of the decays: 1e-5 of the root of the sum of its terms' squares (and of what it is itself)."""
    off = (got.detach().cpu().double() - ref["dg"]).norm().item()
    room = FP32_BAR * max(ref["dg_size"], ref["dg"].norm().item())
    assert off <= room, f"dg: {off:.3e} off, above {room:.1e}"
