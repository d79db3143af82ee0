"""The seam between two blocks and dropout by itself on the GPU, against their definitions in 64 bits."""
import pytest
import torch

from seam_reference import DTYPES, LOW, NAMES, check, factors, inputs, philox, reference

pytestmark = pytest.mark.gpu


def cuda(x):
    return {n: None if t is None else t.cuda() for n, t in x.items()}


def both(x, up, **opts):
    """(Y, H, gradients by name) of the binding's calls."""
    from paper_2602_06935_amd import binding
    g, u = cuda(x), cuda(up)
    vectors = {n: g[n] for n in NAMES[2:]}
    Y, H = binding.cotten_residual_fwd(g["X"], g["F"], **vectors, **opts)
    grads = binding.cotten_residual_bwd(g["X"], g["F"], u["dY"], u["dH"], **vectors, **opts)
    return Y, H, dict(zip(NAMES, grads))


def compare(x, up, **opts):
    ref = reference(x, up, **opts)
    Y, H, grads = both(x, up, **opts)
    check("Y", Y, ref["Y"])
    assert (H is None) == (ref["H"] is None)
    if H is not None:
        check("H", H, ref["H"])
    for n in NAMES:
        assert (grads[n] is None) == (x[n] is None), n
        if x[n] is not None:
            check("gradient of " + n, grads[n], ref[n])


# widths around every change of the lanes that share a row, odd ones, and those that are no multiple of eight
@pytest.mark.parametrize("D", [8, 17, 64, 65, 99, 128, 256, 257, 300, 512, 520, 1000, 2048, 2049, 4096, 4104, 8185, 8192])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_widths(dtype, D):
    for norm, gate in (("layer", "sequence"), ("rms", "channel")):
        x, up = inputs(3, 5, D, DTYPES[dtype], norm=norm, gate=gate, seed=D)
        compare(x, up, norm=norm, alpha=0.7, p=0.25, seed=D * 2 ** 33 + 5, offset=2 ** 40 + D)


@pytest.mark.parametrize("gate", ["none", "channel", "sequence"])
@pytest.mark.parametrize("post,next", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_options(dtype, norm, post, next, gate):
    for p in (0.0, 0.1):
        x, up = inputs(4, 7, 96, DTYPES[dtype], norm=norm, post=post, next=next, gate=gate, seed=3)
        compare(x, up, norm=norm, alpha=-1.3, p=p, seed=9)


@pytest.mark.parametrize("B,N,D", [(1, 1, 64), (700, 1, 64), (3, 4000, 64), (40, 333, 256), (9, 1001, 40), (2, 700, 2048), (5, 200, 3000),
                                   (3, 150, 8190)])
@pytest.mark.parametrize("gate", ["channel", "sequence"])
def test_many_rows(gate, B, N, D):
    """More rows than there are groups of lanes: units of several rows, sequences of several units, the sums over both."""
    x, up = inputs(B, N, D, torch.float32, norm="layer", gate=gate, seed=B + N)
    compare(x, up, norm="layer", alpha=0.5, p=0.1, seed=1)


def test_one_upstream_gradient():
    x, up = inputs(3, 6, 48, torch.float32, gate="channel", seed=4)
    for only in ("dY", "dH"):
        compare(x, {n: t if n == only else None for n, t in up.items()}, norm="layer", p=0.2, seed=3)


@pytest.mark.parametrize("D", [1, 2, 3, 7])
def test_narrow_rows(D):
    """Rows of a value or two: their normalised values are constants, and what is left of gradients through them are
    roundings of what they are made from."""
    x, up = inputs(6, 9, D, torch.float32, norm="rms", gate="channel", seed=D)
    x["X"] = x["X"].sign() * (1.0 + x["X"].abs())
    ref = reference(x, up, norm="rms", alpha=0.1, eps=0.5, p=0.0)
    Y, H, grads = both(x, up, norm="rms", alpha=0.1, eps=0.5)
    check("Y", Y, ref["Y"])
    check("H", H, ref["H"])
    for n in NAMES[:2]:
        assert (grads[n].cpu().double() - ref[n]).abs().max().item() <= 64 * 2.0 ** -24 * 8, n


def test_results_in_place():
    from paper_2602_06935_amd import binding
    for D in (64, 99, 2000):
        x, up = inputs(3, 50, D, torch.bfloat16, gate="channel", seed=D)
        g = cuda(x)
        vectors = {n: g[n] for n in NAMES[2:]}
        Y, H = binding.cotten_residual_fwd(g["X"], g["F"], norm="layer", p=0.3, seed=2, **vectors)
        Y2, H2 = binding.cotten_residual_fwd(g["X"], g["F"], g["X"], g["F"], norm="layer", p=0.3, seed=2, **vectors)
        assert Y2 is g["X"] and H2 is g["F"] and torch.equal(Y, Y2) and torch.equal(H, H2)


def test_what_is_not_finite_stays_in_its_row():
    x, up = inputs(2, 8, 100, torch.float32, seed=5)
    x["F"][0, 3, 7] = float("nan")
    x["F"][1, 2, 50] = float("inf")
    Y, H, grads = both(x, up, norm="layer")
    for t in (Y, H, grads["X"], grads["F"]):
        bad = ~torch.isfinite(t).all(-1)
        assert bad[0, 3] and bad[1, 2] and bad.sum() == 2


def test_dropped_values_may_hold_anything():
    from paper_2602_06935_amd import binding
    f = factors(1000, 0.5, 11, 3)
    x = torch.ones(1000)
    x[f == 0] = float("nan")
    y = binding.cotten_dropout(x.cuda(), 0.5, seed=11, offset=3)
    assert torch.equal(y.cpu().double(), f)
    Y, _ = binding.cotten_residual_fwd(torch.zeros(1, 10, 100).cuda(), x.reshape(1, 10, 100).cuda(), p=0.5, seed=11, offset=3)
    assert torch.equal(Y.cpu().double().flatten(), f)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 4095, 4096, 4097, 100003])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_dropout(dtype, n):
    from paper_2602_06935_amd import binding
    x = torch.randn(n + 24, generator=torch.Generator().manual_seed(n)).to(DTYPES[dtype])
    g = x.cuda()
    for p, seed, offset in ((0.0, 1, 0), (0.1, 0, 2 ** 63 + 1), (0.99, 2 ** 64 - 1, 7)):
        out = g.clone()
        binding.cotten_dropout(g[:n], p, seed=seed, offset=offset, out=out[:n])
        ref = x[:n].double() * factors(n, p, seed, offset)
        got = out[:n].cpu().double()
        # the factor and the product: two roundings of 2^-24, and that of the result: half a step, which below the smallest
        # normal value (fp16: 2^-14, which one value in 16000 is below) is not relative to the value any more (2^-25)
        of_type = torch.finfo(DTYPES[dtype])
        room = ref.abs() * (of_type.eps / 2 + 2.0 ** -23) + of_type.smallest_normal * of_type.eps / 2
        assert ((got - ref).abs() <= room).all()
        assert torch.equal(out[n:], g[n:])                  # what lies behind is left as it was
        same = g.clone()
        binding.cotten_dropout(same[:n], p, seed=seed, offset=offset, out=same[:n])
        assert torch.equal(same, out)


def test_the_seam_drops_what_the_dropout_drops():
    from paper_2602_06935_amd import binding
    for D in (96, 99):
        F = torch.randn(4, 11, D, device="cuda")
        Y, _ = binding.cotten_residual_fwd(torch.zeros_like(F), F, p=0.3, seed=5, offset=6)
        assert torch.equal(Y, binding.cotten_dropout(F, 0.3, seed=5, offset=6))


def test_step_is_added_to_the_offset():
    from paper_2602_06935_amd import binding
    x = torch.randn(5, 40, 64, device="cuda")
    step = torch.tensor([4], device="cuda")
    want = binding.cotten_dropout(x, 0.4, seed=8, offset=7)
    assert torch.equal(want, binding.cotten_dropout(x, 0.4, seed=8, offset=3, step=step))
    assert not torch.equal(want, binding.cotten_dropout(x, 0.4, seed=8, offset=3))
    zero = torch.zeros_like(x)
    assert torch.equal(binding.cotten_residual_fwd(zero, x, p=0.4, seed=8, offset=3, step=step)[0], want)


def test_differentiable_functions():
    from paper_2602_06935_amd import autograd
    opts = dict(norm="layer", alpha=0.7, p=0.2, seed=6, offset=1)
    for gate in ("none", "sequence"):
        x, up = inputs(3, 20, 72, torch.float32, gate=gate, seed=8)
        ref = reference(x, up, **opts)
        leaves = {n: None if t is None else t.cuda().requires_grad_() for n, t in x.items()}
        Y, H = autograd.residual_norm(leaves["X"], leaves["F"], **{n: leaves[n] for n in NAMES[2:]}, **opts)
        loss = (Y * up["dY"].cuda()).sum() + (H * up["dH"].cuda()).sum()
        names = [n for n in NAMES if x[n] is not None]
        for n, t in zip(names, torch.autograd.grad(loss, [leaves[n] for n in names])):
            check(n, t, ref[n])
    X = x["X"].cuda().requires_grad_()
    y = autograd.dropout(X, 0.3, seed=2, offset=9)
    f = factors(X.numel(), 0.3, 2, 9).reshape(X.shape)
    check("dropout", y, x["X"].double() * f)
    dx, = torch.autograd.grad(y, X, up["dY"].cuda())
    check("gradient of the dropout", dx, up["dY"].double() * f)


def test_gradients_against_differences():
    """The loss moves along a direction as its gradient says: what a step of 2^-9 gives, to the third order left out (2^-18) and
    the roundings of the losses (sums of 64-bit products of fp32 results)."""
    from paper_2602_06935_amd import binding
    x, up = inputs(3, 8, 40, torch.float32, gate="sequence", seed=12)
    opts = dict(norm="layer", alpha=0.6, p=0.2, seed=4)
    _, _, grads = both(x, up, **opts)
    gen = torch.Generator().manual_seed(1)
    for n in NAMES:
        way = torch.randn(x[n].shape, generator=gen)
        way /= way.norm()

        def loss(step):
            y = dict(x)
            y[n] = x[n] + step * way
            g = cuda(y)
            Y, H = binding.cotten_residual_fwd(g["X"], g["F"], **{m: g[m] for m in NAMES[2:]}, **opts)
            return ((Y.cpu().double() * up["dY"].double()).sum() + (H.cpu().double() * up["dH"].double()).sum()).item()

        h = 2.0 ** -7
        slope = (loss(h) - loss(-h)) / (2 * h)
        want = (grads[n].cpu().double() * way.double()).sum().item()
        # fp32 roundings of 1920 values of size 1, times upstream values, over the step; and the third derivative
        room = (1920 ** 0.5 * 2.0 ** -24 * 4) / h + 64 * h * h
        assert abs(slope - want) <= room, (n, slope, want)


def test_large_offsets():
    """More than 2^32 elements dropped, and more than 2^32 bytes of rows: the last ones, and their numbers."""
    from paper_2602_06935_amd import binding
    n = 2 ** 32 + 12345
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    binding.cotten_dropout(x, 0.25, seed=5, offset=1, out=x)
    first = 2 ** 32 - 40000 + 40000 % 8
    group = torch.arange(first // 8, (n + 7) // 8).tolist()
    words = [philox([g & LOW, g >> 32, 1, 0], (5, 0)) for g in group[-200:]]
    lots = [h for w in words for c in w for h in (c & 0xffff, c >> 16)]
    at = group[-200] * 8
    want = torch.tensor([4 / 3 if h >= 16384 else 0.0 for h in lots])[:n - at].to(torch.bfloat16)
    assert torch.equal(x[at:].cpu(), want)
    del x
    X = torch.zeros(1100, 1000, 2040, dtype=torch.bfloat16, device="cuda")
    assert X.numel() > 2 ** 31
    X[-1, -1] = torch.randn(2040, device="cuda").to(torch.bfloat16)
    weight = torch.ones(2040, dtype=torch.bfloat16, device="cuda")
    Y, H = binding.cotten_residual_fwd(X, X, X, next_weight=weight, alpha=1.0)
    small = torch.zeros(1, 1, 2040, dtype=torch.bfloat16, device="cuda")
    small[0, 0] = Y[-1, -1] / 2
    again = binding.cotten_residual_fwd(small, small, next_weight=weight)
    assert torch.equal(Y[-1:, -1:], again[0]) and torch.equal(H[-1:, -1:], again[1])


def test_runs_are_alike():
    x, up = inputs(33, 70, 136, torch.bfloat16, gate="sequence", seed=7)
    opts = dict(norm="layer", p=0.1, seed=3)
    first, again = both(x, up, **opts), both(x, up, **opts)
    for a, b in zip((*first[:2], *first[2].values()), (*again[:2], *again[2].values())):
        assert torch.equal(a, b)


def test_on_another_stream():
    from paper_2602_06935_amd import binding
    x, up = inputs(3, 30, 64, torch.float32, seed=2)
    ref = reference(x, up, norm="layer")
    g, u = cuda(x), cuda(up)
    vectors = {n: g[n] for n in NAMES[2:]}
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    Y, H = binding.cotten_residual_fwd(g["X"], g["F"], norm="layer", stream=s, **vectors)
    grads = binding.cotten_residual_bwd(g["X"], g["F"], u["dY"], u["dH"], norm="layer", stream=s, **vectors)
    s.synchronize()
    check("Y", Y, ref["Y"])
    check("H", H, ref["H"])
    for n, t in zip(NAMES, grads):
        if t is not None:
            check(n, t, ref[n])


def test_captured():
    """Replays follow the inputs and, by `step`, the generator."""
    from paper_2602_06935_amd import binding
    x, up = inputs(4, 60, 256, torch.bfloat16, gate="sequence", seed=6)
    g, u = cuda(x), cuda(up)
    vectors = {n: g[n] for n in NAMES[2:]}
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    opts = dict(norm="layer", p=0.2, seed=3, **vectors)

    def calls(**kw):
        Y, H = binding.cotten_residual_fwd(g["X"], g["F"], **opts, **kw)
        return (Y, H, *binding.cotten_residual_bwd(g["X"], g["F"], u["dY"], u["dH"], **opts, **kw),
                binding.cotten_dropout(Y, 0.5, seed=3, **kw))

    calls(step=step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls(step=step)
    for i in range(4):
        step.fill_(i)
        g["F"].mul_(-0.9)
        graph.replay()
        want = calls(offset=i)
        torch.cuda.synchronize()
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(got, want)), i
