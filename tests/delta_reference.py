"""The gated delta rule from its definition, token by token in 64 bits on the CPU, with gradients by differentiating
that; inputs for the tests; how far a result may be from it.

Bounds.  Nothing is rounded below 24 significant bits before a result is stored, so a fp32 result carries the fp32
rounding errors (2^-24 each) of the sums of d + 32 products that make it, of the few such sums in a row that lead from an
input to it, and of the chunks before it, which decays and corrections damp: sqrt(160) * 2^-24 * 8, below 1e-5.  A
16-bit result is off by its own rounding besides, at most eps / 2 of every value."""
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FP32_BAR = 1e-5
ROW_FACTOR = 4.0     # rows: against the larger of their own and the tensor's typical row


def bar_for(dtype):
    return FP32_BAR + (0.0 if dtype is torch.float32 else torch.finfo(dtype).eps / 2)


def check(name, got, ref):
    got64, ref = got.detach().cpu().double(), ref.double()
    assert got64.shape == ref.shape, name
    assert torch.isfinite(got64).all(), f"{name}: not finite"
    bar = bar_for(got.dtype)
    diff, norm = (got64 - ref).norm().item(), ref.norm().item()
    assert diff <= bar * norm, f"{name}: {diff / max(norm, 1e-300):.3e} off, above {bar:.1e}"
    if norm > 0:
        rows = (got64 - ref).reshape(-1, ref.shape[-1]).norm(dim=-1)
        own = ref.reshape(-1, ref.shape[-1]).norm(dim=-1)
        typical = (own.square().mean()).sqrt()
        worst = (rows / torch.maximum(own, typical)).max().item()
        assert worst <= ROW_FACTOR * bar, f"{name}: a row {worst:.3e} off, above {ROW_FACTOR * bar:.1e}"


def inputs(B, H, N, d, dtype, seed=0, mask=None, states=False):
    """CPU tensors in [B,H,N,...] order, floats rounded to `dtype` where the operator takes that type."""
    gen = torch.Generator().manual_seed(seed)
    x = {}
    for n in ("q", "k", "v", "dO"):
        x[n] = torch.randn(B, H, N, d, generator=gen).to(dtype)
    x["g"] = -torch.exp((torch.rand(B, H, N, generator=gen) - 1.0) * 7.0)
    x["beta"] = torch.sigmoid(1.5 * torch.randn(B, H, N, generator=gen))
    x["mask"] = None
    if mask is not None:
        lengths = torch.randint(1, N + 1, (B,), generator=gen)
        m = torch.arange(N)[None, :] >= (N - lengths)[:, None]            # histories padded on the left
        if mask == "holes":
            m = torch.rand(B, N, generator=gen) < 0.6
        if mask in ("holes", "empty"):
            m[-1] = False                                                 # a sequence without any valid token
        x["mask"] = m.to(torch.uint8)
    x["S0"] = torch.randn(B, H, d, d, generator=gen) * 0.3 if states else None
    x["dS1"] = torch.randn(B, H, d, d, generator=gen) * 0.3 if states else None
    return x


def reference(x, scale=1.0, eps=1e-6, grads=True):
    """O, S1 and, with `grads`, dQ, dK, dV, dg, dbeta, dS0 (all [B,H,N,...], float64)."""
    q, k, v, g, beta = (x[n].detach().double() for n in ("q", "k", "v", "g", "beta"))
    B, H, N, d = q.shape
    if x["mask"] is not None:   # what masked rows hold is never looked at
        live = x["mask"].bool()[:, None, :].expand(B, H, N)
        k, v = (torch.where(live[..., None], t, torch.zeros(())) for t in (k, v))
        g, beta = (torch.where(live, t, torch.zeros(())) for t in (g, beta))
    S0 = torch.zeros(B, H, d, d, dtype=torch.float64) if x["S0"] is None else x["S0"].double().clone()
    leaves = [t.clone().requires_grad_(grads) for t in (q, k, v, g, beta, S0)]
    q, k, v, g, beta, S = leaves
    if x["mask"] is not None:
        g, beta = g * live, beta * live
    qn = q / (q.square().sum(-1, keepdim=True) + eps).sqrt()
    kk = k.square().sum(-1, keepdim=True) + eps
    if x["mask"] is not None:
        kk = torch.where(live[..., None], kk, torch.ones((), dtype=torch.float64))   # (rows of zeros, whatever eps is)
    kn = k / kk.sqrt()
    o = []
    for t in range(N):
        S = g[:, :, t, None, None].exp() * S
        e = v[:, :, t] - torch.einsum("bha,bhac->bhc", kn[:, :, t], S)
        S = S + torch.einsum("bha,bhc->bhac", kn[:, :, t], beta[:, :, t, None] * e)
        o.append(scale * torch.einsum("bha,bhac->bhc", qn[:, :, t], S))
    O = torch.stack(o, 2)
    out = {"O": O.detach(), "S1": S.detach()}
    if grads:
        loss = (O * x["dO"].double()).sum()
        if x["dS1"] is not None:
            loss = loss + (S * x["dS1"].double()).sum()
        got = torch.autograd.grad(loss, leaves)
        out.update(zip(("dQ", "dK", "dV", "dg", "dbeta", "dS0"), got))
        if x["mask"] is not None:
            for n in ("dK", "dV", "dg", "dbeta"):
                out[n] = torch.where(live if out[n].dim() == 3 else live[..., None], out[n], torch.zeros((), dtype=torch.float64))
    return out
