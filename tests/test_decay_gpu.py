"""The decay attention on the GPU, forward, backward and single steps, against its definition in 64 bits."""
import math

import pytest
import torch

from decay_reference import DTYPES, FP32_BAR, check, check_decays, inputs, reference

pytestmark = pytest.mark.gpu

NAMES = ("dQ", "dK", "dV")


def lay(t, layout):
    return t.cuda() if layout == "bhnd" else t.transpose(1, 2).contiguous().cuda()


def back(t, layout):
    return t if layout == "bhnd" else t.transpose(1, 2)


def cuda(t):
    return None if t is None else t.cuda()


def forward(x, layout="bhnd", scale=1.0, **kw):
    from paper_2602_06935_amd import binding
    q, k, v = (lay(x[n], layout) for n in ("q", "k", "v"))
    B, H, N, d = x["q"].shape
    S1 = torch.empty(B, H, d, d, device="cuda")
    O = binding.cotten_decay_fwd(q, k, v, x["g"].cuda(), cuda(x["mask"]), scale=scale, layout=layout,
                                 initial_state=cuda(x["S0"]), final_state=S1, **kw)
    return back(O, layout), S1


def backward(x, layout="bhnd", scale=1.0, decays=True, **kw):
    from paper_2602_06935_amd import binding
    q, k, v, dO = (lay(x[n], layout) for n in ("q", "k", "v", "dO"))
    B, H, N, d = x["q"].shape
    dS0 = torch.empty(B, H, d, d, device="cuda")
    dg = torch.empty(H, device="cuda") if decays else None
    grads = binding.cotten_decay_bwd(q, k, v, x["g"].cuda(), cuda(x["mask"]), dO, dg=dg, scale=scale, layout=layout,
                                     initial_state=cuda(x["S0"]), dfinal_state=cuda(x["dS1"]), dinitial_state=dS0, **kw)
    return dict(zip(NAMES, (back(t, layout) for t in grads)), dS0=dS0, dg=dg)


def compare(x, layout="bhnd", scale=1.0, grads=True):
    ref = reference(x, scale=scale, grads=grads)
    O, S1 = forward(x, layout, scale)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])
    if grads:
        got = backward(x, layout, scale)
        for n in NAMES + ("dS0",):
            check(n, got[n], ref[n])
        check_decays(got["dg"], ref)
        plain = backward(x, layout, scale, decays=False)
        assert all(torch.equal(got[n], plain[n]) for n in NAMES + ("dS0",))
        if x["mask"] is not None:
            off = (x["mask"] == 0)[:, None, :].expand(x["q"].shape[:3]).cuda()
            assert (got["dK"][off] == 0).all() and (got["dV"][off] == 0).all()
    return ref


# lengths around those of the recurrence, of a chunk and of two
@pytest.mark.parametrize("N", [1, 2, 5, 6, 7, 10, 11, 12, 13, 31, 32, 33, 63, 65, 100])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_lengths(dtype, d, N):
    compare(inputs(2, 3, N, d, DTYPES[dtype], seed=N + d, mask="left" if N > 1 else None, states=N % 2 == 1), scale=0.5)


@pytest.mark.parametrize("mask", [None, "left", "right", "holes", "empty"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_masks_and_layouts(dtype, d, layout, mask):
    compare(inputs(3, 2, 77, d, DTYPES[dtype], seed=d, mask=mask, states=True), layout)


@pytest.mark.parametrize("N", [3, 50])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_without_states(dtype, N):
    from paper_2602_06935_amd import binding
    x = inputs(2, 2, N, 32, DTYPES[dtype], seed=7)
    ref = reference(x)
    q, k, v, dO = (x[n].cuda() for n in ("q", "k", "v", "dO"))
    O = binding.cotten_decay_fwd(q, k, v, x["g"].cuda(), None)
    check("O", O, ref["O"])
    for n, t in zip(NAMES, binding.cotten_decay_bwd(q, k, v, x["g"].cuda(), None, dO)):
        check(n, t, ref[n])


# sequences long enough, and few enough, to be cut into segments
@pytest.mark.parametrize("B,H,N,d", [(1, 1, 1500, 64), (1, 2, 1100, 128), (2, 2, 900, 32), (1, 3, 1000, 16)])
@pytest.mark.parametrize("mask,layout", [("left", "bnhd"), ("holes", "bhnd")])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_segments(dtype, mask, layout, B, H, N, d):
    from paper_2602_06935_amd import binding
    assert binding.cotten_decay_workspace_bytes(B, H, N, d, 1, False) > 0 and binding.cotten_decay_workspace_bytes(B, H, N, d, 1, True) > 0
    x = inputs(B, H, N, d, DTYPES[dtype], seed=N, mask=mask, states=True)
    if mask == "holes" and B == 1:
        x["mask"][0, 400:] = 1                       # a stretch without holes, and one without tokens
        x["mask"][0, 200:300] = 0
    compare(x, layout, scale=0.25)


# few segments, which find the states before them themselves; also where the state is replaced in place
@pytest.mark.parametrize("B,H,N,d", [(1, 2, 400, 64), (2, 1, 330, 128), (1, 3, 390, 32), (1, 1, 330, 16)])
@pytest.mark.parametrize("mask", [None, "left", "holes"])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_few_segments(dtype, mask, B, H, N, d):
    from paper_2602_06935_amd import binding
    segments = binding.cotten_decay_workspace_bytes(B, H, N, d, binding._DTYPE_CODES[DTYPES[dtype]], False) // (4 * B * H * d * d)
    assert 3 <= segments <= 6
    x = inputs(B, H, N, d, DTYPES[dtype], seed=N + d, mask=mask, states=True)
    ref = compare(x, "bnhd", scale=0.25)
    q, k, v, g, state = (x[n].cuda() for n in ("q", "k", "v", "g", "S0"))
    O = binding.cotten_decay_fwd(q, k, v, g, cuda(x["mask"]), scale=0.25, initial_state=state, final_state=state)
    check("O", O, ref["O"])
    check("S1", state, ref["S1"])


# numbers of slices (and of segments) for which keys' and values' gradients are one walk: 86 ... 128, 342 ... 384 at d = 128
@pytest.mark.parametrize("B,H,N", [(29, 3, 33), (64, 2, 70), (43, 2, 64), (49, 7, 40), (16, 1, 520)])
@pytest.mark.parametrize("mask", [None, "left", "right", "holes", "empty"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_joint_gradients(dtype, mask, B, H, N):
    x = inputs(B, H, N, 128, DTYPES[dtype], seed=B + N, mask=mask, states=mask != "left")
    compare(x, "bnhd" if N % 2 else "bhnd", scale=0.25)


@pytest.mark.parametrize("d,B,H", [(64, 293, 7), (128, 150, 3), (16, 700, 2), (32, 520, 4)])
@pytest.mark.parametrize("N", [1, 3, 40])
def test_many_slices(N, d, B, H):
    for dtype in ("f32", "bf16"):
        x = inputs(B, H, N, d, DTYPES[dtype], seed=60 + d + N, mask="holes" if N > 1 else None, states=True)
        compare(x, "bnhd", grads=N == 40 and d <= 32)


@pytest.mark.parametrize("N", [1, 4, 70, 700])
def test_states_are_replaced_in_place(N):
    """A server's state: also where other workgroups start from it (segments)."""
    from paper_2602_06935_amd import binding
    x = inputs(1, 2, N, 64, torch.bfloat16, seed=N, states=True)
    S = x["S0"].cuda()
    q, k, v, g = (x[n].cuda() for n in ("q", "k", "v", "g"))
    O, S1 = forward(x)
    O2 = binding.cotten_decay_fwd(q, k, v, g, None, initial_state=S, final_state=S)
    assert torch.equal(O, O2) and torch.equal(S, S1)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_steps_follow_the_whole_sequence(dtype, d):
    """Token by token, and in parts of 1 ... 40 tokens, from the states handed over: what one call makes of all."""
    from paper_2602_06935_amd import binding
    x = inputs(2, 2, 97, d, DTYPES[dtype], seed=d, mask="left", states=True)
    ref = reference(x, grads=False)
    for cuts in (list(range(98)), [0, 1, 4, 8, 40, 57, 97]):
        S, O = x["S0"].cuda(), []
        for a, b in zip(cuts, cuts[1:]):
            q, k, v = (x[n][:, :, a:b].contiguous().cuda() for n in ("q", "k", "v"))
            O.append(binding.cotten_decay_fwd(q, k, v, x["g"].cuda(), x["mask"][:, a:b].contiguous().cuda(), initial_state=S, final_state=S))
        check("O", torch.cat(O, 2), ref["O"])
        # (a rounding of the state by every call)
        assert (S.cpu().double() - ref["S1"]).norm() <= FP32_BAR * ref["S1"].norm()


@pytest.mark.parametrize("N", [4, 90, 1200])
@pytest.mark.parametrize("rate", [0.0, -1e-5, -30.0, -200.0, float("-inf"), 0.01])
def test_rates(rate, N):
    """No decay (the causal attention), a weak one, decays to nothing within a token, and growth."""
    x = inputs(1, 2, N, 32, torch.float32, seed=11, mask="holes" if N == 90 else None, states=True)
    if x["mask"] is not None:
        x["mask"][0] = (torch.rand(N, generator=torch.Generator().manual_seed(2)) < 0.7).to(torch.uint8)
    x["g"] = torch.tensor([rate, -0.05])
    if rate == float("-inf"):
        # exp(-inf) * S: the definition's derivative by g is 0 * inf
        ref = reference(dict(x, g=torch.tensor([-1e5, -0.05], dtype=torch.float64)))
        O, S1 = forward(x)
        check("O", O, ref["O"])
        check("S1", S1, ref["S1"])
        got = backward(x)
        for n in NAMES + ("dS0",):
            check(n, got[n], ref[n])
        check_decays(got["dg"], ref)
    else:
        compare(x, scale=0.5)


def test_no_decay_is_the_causal_attention():
    from paper_2602_06935_amd import binding
    x = inputs(2, 2, 300, 64, torch.float32, seed=3)
    q, k, v = (x[n].cuda() for n in ("q", "k", "v"))
    O = binding.cotten_decay_fwd(q, k, v, torch.zeros(2, device="cuda"), None, scale=1 / 300)
    check("O", O, binding.cotten_attn_fwd(q, k, v, None, causal=True).cpu())


def test_what_masked_rows_hold_is_not_looked_at():
    for N in (4, 70, 900):
        x = inputs(1, 2, N, 64, torch.bfloat16, seed=N, states=True)
        x["mask"] = (torch.rand(1, N, generator=torch.Generator().manual_seed(N)) < 0.5).to(torch.uint8)
        off = (x["mask"] == 0)[0]
        dirty = {n: t for n, t in x.items()}
        for n, v in (("k", float("nan")), ("v", float("inf"))):
            dirty[n] = x[n].clone()
            dirty[n][:, :, off] = v
        clean = forward(x) + tuple(backward(x).values())
        got = forward(dirty) + tuple(backward(dirty).values())
        assert all(torch.equal(a, b) for a, b in zip(clean, got))


def test_values_that_are_not_finite_stay_in_their_sequence():
    x = inputs(3, 2, 90, 32, torch.float32, seed=5, states=True)
    clean = forward(x)
    x["v"][1, 0, 40, 3] = float("nan")
    O, S1 = forward(x)
    assert torch.isnan(O[1, 0, 40:, 3]).all() and torch.isfinite(O[1, 0, :32]).all()
    keep = torch.ones(3, 2, dtype=torch.bool)
    keep[1, 0] = False
    assert torch.equal(O[keep.cuda()], clean[0][keep.cuda()]) and torch.equal(S1[keep.cuda()], clean[1][keep.cuda()])


@pytest.mark.parametrize("N", [1, 40, 1000])
def test_runs_are_alike(N):
    x = inputs(2, 2, N, 64, torch.bfloat16, seed=N, mask="left" if N > 1 else None, states=True)
    first, again = forward(x) + tuple(backward(x).values()), forward(x) + tuple(backward(x).values())
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_differentiable_function(dtype):
    from paper_2602_06935_amd.autograd import decay_attention
    for layout in ("bhnd", "bnhd"):
        x = inputs(2, 3, 75, 32, DTYPES[dtype], seed=9, mask="left", states=True)
        ref = reference(x, scale=0.3)
        q, k, v = (lay(x[n], layout).requires_grad_() for n in ("q", "k", "v"))
        g, S0 = x["g"].cuda().requires_grad_(), x["S0"].cuda().requires_grad_()
        O, S1 = decay_attention(q, k, v, g, x["mask"].cuda(), scale=0.3, layout=layout, initial_state=S0, return_state=True)
        grads = torch.autograd.grad([O, S1], [q, k, v, g, S0], [lay(x["dO"], layout), x["dS1"].cuda()])
        check("O", back(O, layout), ref["O"])
        check("S1", S1, ref["S1"])
        for n, t in zip(NAMES, grads):
            check(n, back(t, layout), ref[n])
        check_decays(grads[3], ref)
        check("dS0", grads[4], ref["dS0"])
        # the state alone, and decays that want no gradient
        O, S1 = decay_attention(q, k, v, g.detach(), x["mask"].cuda(), scale=0.3, layout=layout, return_state=True)
        dk, = torch.autograd.grad(S1, k, x["dS1"].cuda())
        check("dK", back(dk, layout), reference(dict(x, S0=None, dO=torch.zeros_like(x["dO"])), scale=0.3)["dK"])


def test_gradients_against_differences():
    """The loss moves along a direction as its gradient says, but for the third order of the step and the roundings of fp32 outputs."""
    x = inputs(1, 2, 70, 32, torch.float32, seed=4, mask="holes", states=True)
    x["mask"][0] = (torch.rand(70, generator=torch.Generator().manual_seed(1)) < 0.7).to(torch.uint8)
    got = backward(x)
    gen = torch.Generator().manual_seed(2)

    def loss(y):
        O, S1 = forward(y)
        return ((O.cpu().double() * x["dO"].double()).sum() + (S1.cpu().double() * x["dS1"].double()).sum()).item()

    h = 2.0 ** -6
    for n, of in (("q", "dQ"), ("k", "dK"), ("v", "dV"), ("g", "dg"), ("S0", "dS0")):
        way = torch.randn(x[n].shape, generator=gen)
        way /= way.norm()
        slope = (loss(dict(x, **{n: x[n] + h * way})) - loss(dict(x, **{n: x[n] - h * way}))) / (2 * h)
        want = (got[of].cpu().double() * way.double()).sum().item()
        # 6500 outputs of size 1, off by a few 2^-24 each, times upstream values, over the step; and the third derivative
        room = (6528 ** 0.5 * 2.0 ** -24 * 8) / h + 4 * h * h * max(1.0, got[of].cpu().double().norm().item())
        assert abs(slope - want) <= room, (n, slope, want)


def test_large_offsets():
    """Tensors of more than 2^32 bytes: the last sequences are as they are by themselves."""
    from paper_2602_06935_amd import binding
    x = inputs(2, 3, 300, 128, torch.float32, seed=21, mask="left")
    B = 9500
    big = {n: torch.zeros(B, 300, 3, 128, device="cuda") for n in ("q", "k", "v", "dO")}
    assert big["q"].numel() * 4 > 2 ** 32
    for n, t in big.items():
        t[-2:] = lay(x[n], "bnhd")
    mask = torch.ones(B, 300, dtype=torch.uint8, device="cuda")
    mask[-2:] = x["mask"].cuda()
    g = x["g"].cuda()
    O, S1 = forward(x, "bnhd")
    got = binding.cotten_decay_fwd(big["q"], big["k"], big["v"], g, mask, layout="bnhd")
    assert torch.equal(back(got, "bnhd")[-2:], O)
    del got
    want = backward(x, "bnhd", decays=False)
    grads = binding.cotten_decay_bwd(big["q"], big["k"], big["v"], g, mask, big["dO"], layout="bnhd")
    for n, t in zip(NAMES, grads):
        check(n, back(t, "bnhd")[-2:], want[n].cpu())


def test_on_another_stream_and_with_a_given_workspace():
    from paper_2602_06935_amd import binding
    x = inputs(1, 2, 800, 64, torch.float32, seed=13, states=True)
    ref = reference(x)
    q, k, v, dO, g = (x[n].cuda() for n in ("q", "k", "v", "dO", "g"))
    S0, dS1, S1, dg = x["S0"].cuda(), x["dS1"].cuda(), torch.empty(1, 2, 64, 64, device="cuda"), torch.empty(2, device="cuda")
    spaces = [torch.full((binding.cotten_decay_workspace_bytes(1, 2, 800, 64, 0, b, b),), 255, dtype=torch.uint8, device="cuda") for b in (False, True)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    O = binding.cotten_decay_fwd(q, k, v, g, None, stream=s, initial_state=S0, final_state=S1, workspace=spaces[0])
    grads = binding.cotten_decay_bwd(q, k, v, g, None, dO, dg=dg, stream=s, initial_state=S0, dfinal_state=dS1, workspace=spaces[1])
    s.synchronize()
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])
    for n, t in zip(NAMES, grads):
        check(n, t, ref[n])
    check_decays(dg, ref)


def test_captured():
    from paper_2602_06935_amd import binding
    x = inputs(2, 2, 400, 64, torch.bfloat16, seed=15, mask="left", states=True)
    q, k, v, dO, g = (x[n].cuda() for n in ("q", "k", "v", "dO", "g"))
    mask, S0, dS1 = x["mask"].cuda(), x["S0"].cuda(), x["dS1"].cuda()
    step = [t[:, :, :1].contiguous() for t in (q, k, v)]
    state = S0.clone()

    def calls():
        S1, dg = torch.empty_like(S0), torch.empty_like(g)
        O = binding.cotten_decay_fwd(q, k, v, g, mask, initial_state=S0, final_state=S1)
        grads = binding.cotten_decay_bwd(q, k, v, g, mask, dO, dg=dg, initial_state=S0, dfinal_state=dS1)
        return (O, S1, dg, *grads, binding.cotten_decay_fwd(*step, g, None, initial_state=state, final_state=state))

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for i in range(4):
        v.mul_(-0.7)
        g.mul_(1.1)
        state.copy_(S0 * i)
        graph.replay()
        after = state.clone()
        state.copy_(S0 * i)
        want = calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, after), (*want, state))), i


def mixed_masks(N):
    """One sequence each: padded on the right, live tokens on either side of a stretch without any, padded on the left over more than half
    of its length, live at its first token alone, without a live token."""
    m = torch.zeros(5, N, dtype=torch.uint8)
    m[0, :N // 5] = 1
    m[1, :N // 6] = 1
    m[1, 2 * N // 3:] = 1
    m[2, 3 * N // 5:] = 1
    m[3, 0] = 1
    return m


# segments that begin with masked tokens, where nothing comes in from outside and nobody asks for the gradient of that: rows of Q and dO count there
@pytest.mark.parametrize("H,N,d", [(1, 400, 64), (1, 1500, 64), (2, 1100, 128), (1, 330, 128), (2, 900, 32), (1, 390, 32), (1, 1000, 16)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_masked_beginnings_of_segments(dtype, H, N, d):
    from paper_2602_06935_amd import binding
    from paper_2602_06935_amd.autograd import decay_attention
    code = binding._DTYPE_CODES[DTYPES[dtype]]
    for bwd in (False, True):
        assert binding.cotten_decay_workspace_bytes(5, H, N, d, code, bwd) > 0
    layout = "bnhd" if N % 4 else "bhnd"
    x = inputs(5, H, N, d, DTYPES[dtype], seed=N + d, rates=(1e-3, 1e-1))
    x["mask"] = mixed_masks(N)
    ref = reference(x, scale=0.25)
    q, k, v = (lay(x[n], layout).requires_grad_() for n in ("q", "k", "v"))
    g = x["g"].cuda().requires_grad_()
    O = decay_attention(q, k, v, g, x["mask"].cuda(), scale=0.25, layout=layout)
    grads = torch.autograd.grad(O, [q, k, v, g], lay(x["dO"], layout))
    got = dict(zip(NAMES, (back(t, layout) for t in grads)), O=back(O.detach(), layout))
    for n in ("O",) + NAMES:
        for b in range(5):                      # (each sequence by itself: a small one's error is not lost in the others')
            if ref[n][b].any():
                check(f"{n}[{b}]", got[n][b], ref[n][b])
            else:
                assert not got[n][b].any(), (n, b)
    check_decays(grads[3], ref)
    # a state of zeros is no state, and a gradient that comes in behind the sequence changes nothing of what is skipped
    zeros = torch.zeros(5, H, d, d, device="cuda")
    check("O", back(binding.cotten_decay_fwd(q.detach(), k.detach(), v.detach(), g.detach(), x["mask"].cuda(), scale=0.25, layout=layout,
                                             initial_state=zeros), layout), ref["O"])
    x["dS1"] = torch.randn(5, H, d, d, generator=torch.Generator().manual_seed(d)) * 0.3
    ref = reference(x, scale=0.25)
    dg = torch.empty(H, device="cuda")
    grads = binding.cotten_decay_bwd(q.detach(), k.detach(), v.detach(), g.detach(), x["mask"].cuda(), lay(x["dO"], layout), dg=dg, scale=0.25,
                                     layout=layout, dfinal_state=x["dS1"].cuda())
    for n, t in zip(NAMES, grads):
        check(n, back(t, layout), ref[n])
    check_decays(dg, ref)


@pytest.mark.parametrize("N,mask", [(20, None), (40, "left"), (420, "left"), (420, "few")])
@pytest.mark.parametrize("d", [16, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_growth_between_tokens_that_do_not_count(dtype, d, N, mask):
    """A state that grows by e^3 with every token that counts: e^93 of the pairs that are 31 tokens apart is above what fp32 holds, but of such
    pairs one token here does not count or does not exist."""
    x = inputs(2, 2, N, d, DTYPES[dtype], seed=N + d)
    x["g"] = torch.tensor([3.0, -0.1])
    if mask is not None:
        x["mask"] = torch.zeros(2, N, dtype=torch.uint8)
        x["mask"][:, -6:] = 1                                     # the last of a chunk that begins with none
        if mask == "few":
            x["mask"][0, 5:200:40] = 1
    compare(x, scale=0.5)


@pytest.mark.parametrize("tokens", [1, 4])
def test_many_steps_of_a_weak_decay(tokens):
    """exp(g) as one float is off by up to 2^-25, in the same direction at every token: over 3000 of them the oldest would be off by 9e-5.  The
    roundings of the state, one a token, are of either sign."""
    from paper_2602_06935_amd import binding
    N, d = 3000, 16
    x = inputs(1, 4, N, d, torch.float32, seed=tokens)
    # decays half way between two floats, the closest that a float g comes to them
    x["g"] = torch.tensor([math.log1p(-(m + 0.5) * 2.0 ** -24) for m in (200, 1677, 1678, 8000)]).float()
    ref = reference(x, grads=False)
    S, O = torch.zeros(1, 4, d, d, device="cuda"), []
    q, k, v = (torch.stack(x[n].split(tokens, 2)).cuda() for n in ("q", "k", "v"))
    g = x["g"].cuda()
    for i in range(N // tokens):
        O.append(binding.cotten_decay_fwd(q[i], k[i], v[i], g, None, initial_state=S, final_state=S))
    for h in range(4):
        assert (S.cpu().double() - ref["S1"])[:, h].norm() <= FP32_BAR * ref["S1"][:, h].norm(), h
    check("O", torch.cat(O, 2), ref["O"])


# forwards of many segments of narrow states: with all compute units busy, and few slices of long sequences
@pytest.mark.parametrize("B,H,N,d", [(32, 2, 1100, 32), (2, 1, 20000, 32), (4, 1, 16500, 32), (1, 1, 40000, 16)])
def test_forwards_of_many_segments(B, H, N, d):
    for dtype in ("f32", "bf16"):
        x = inputs(B, H, N, d, DTYPES[dtype], seed=N, mask="left" if B > 1 else None, states=True)
        ref = reference(x, grads=False)
        O, S1 = forward(x, "bnhd")
        check("O", O, ref["O"])
        check("S1", S1, ref["S1"])
