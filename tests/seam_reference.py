"""Dropout and the seam between two blocks from their definitions: the generator with Python's own whole numbers, norms, gates
and sums in 64 bits on the CPU, gradients by differentiating that; how far a result may be from it.

Bounds.  A value of Y is four roundings of 2^-24 from the formula; one of H or of a gradient passes the norms as well, sums of D
terms made by lanes and then over these (the longest chain is some 40 additions, errors add up as their root), and sums over
rows one or two more chains of up to a hundred: below 64 * 2^-24 of the tensor's typical value.  A 16-bit result is off by its
own rounding besides, eps / 2 of every value at most."""
import numpy
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FP32_BAR = 64 * 2.0 ** -24
LOW = 0xffffffff


def philox(counter, key):
    c, (k0, k1) = list(counter), key
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k0, b & LOW, (a >> 32) ^ c[3] ^ k1, a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return c


def factors(n, p, seed, offset):
    """0, or one over the share that is kept, for elements 0 ... n-1."""
    out_of = int(numpy.floor(p * 65536 + 0.5))
    group = numpy.arange((n + 7) // 8, dtype=object)
    c = [group & LOW, group >> 32, group * 0 + (offset & LOW), group * 0 + (offset >> 32)]
    words = philox(c, (seed & LOW, seed >> 32))
    lots = numpy.stack([h for w in words for h in (w & 0xffff, w >> 16)], 1).reshape(-1)[:n].astype(numpy.int64)
    return torch.from_numpy(numpy.where(lots >= out_of, 65536.0 / (65536 - out_of), 0.0))


def check(name, got, ref, bar=FP32_BAR):
    got64, ref = got.detach().cpu().double(), ref.double()
    assert got64.shape == ref.shape, name
    assert torch.isfinite(got64).all(), f"{name}: not finite"
    half_step = 0.0 if got.dtype is torch.float32 else torch.finfo(got.dtype).eps / 2
    typical = ref.square().mean().sqrt().item()
    diff = (got64 - ref).abs()
    assert diff.square().mean().sqrt().item() <= (bar + half_step) * typical, f"{name}: {(diff.square().mean().sqrt() / typical).item():.2e}"
    # every value: its own rounding, and eight times the bar for the largest of many errors
    worst = (diff - half_step * ref.abs()).max().item()
    assert worst <= 8 * bar * max(typical, ref.abs().max().item() / 8), f"{name}: a value {worst / typical:.2e} off"


def inputs(B, N, D, dtype, *, norm="layer", post=True, next=True, gate="none", seed=0):
    gen = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=gen) * scale + mean).to(dtype)

    layer = norm == "layer"
    x = dict(X=normal(B, N, D), F=normal(B, N, D, scale=0.7, mean=0.2))
    x["post_weight"] = normal(D, scale=0.2, mean=1.0) if post else None
    x["post_bias"] = normal(D, scale=0.1) if post and layer else None
    x["gate"] = {"none": None, "channel": normal(D, scale=0.3, mean=0.5), "sequence": normal(B, D, scale=0.3, mean=0.5)}[gate]
    x["next_weight"] = normal(D, scale=0.2, mean=1.0) if next else None
    x["next_bias"] = normal(D, scale=0.1) if next and layer else None
    up = dict(dY=normal(B, N, D), dH=normal(B, N, D) if next else None)
    return x, up


NAMES = ("X", "F", "post_weight", "post_bias", "gate", "next_weight", "next_bias")


def reference(x, up, *, norm, alpha=1.0, eps=1e-6, p=0.0, seed=0, offset=0):
    """Y, H and, by the name of what they belong to, the gradients."""
    t = {n: None if v is None else v.detach().double().requires_grad_() for n, v in x.items()}

    def normalised(v, w, b):
        if norm == "layer":
            v = v - v.mean(-1, keepdim=True)
        v = v / (v.square().mean(-1, keepdim=True) + eps).sqrt() * w
        return v if b is None else v + b

    z = t["F"]
    if t["post_weight"] is not None:
        z = normalised(z, t["post_weight"], t["post_bias"])
    if p > 0:
        f = factors(z.numel(), p, seed, offset).reshape(z.shape)
        z = torch.where(f > 0, z * f, 0.0)
    if t["gate"] is not None:
        z = z * (t["gate"] if t["gate"].dim() == 1 else t["gate"][:, None, :])
    Y = t["X"] + alpha * z
    H = None if t["next_weight"] is None else normalised(Y, t["next_weight"], t["next_bias"])
    out = {"Y": Y.detach(), "H": None if H is None else H.detach()}
    pairs = [(o, up[n].double()) for o, n in ((Y, "dY"), (H, "dH")) if o is not None and up.get(n) is not None]
    if pairs:
        names = [n for n in NAMES if t[n] is not None]
        grads = torch.autograd.grad([o for o, _ in pairs], [t[n] for n in names], [g for _, g in pairs], allow_unused=True)
        out.update((n, torch.zeros_like(t[n]) if g is None else g) for n, g in zip(names, grads))
    return out
