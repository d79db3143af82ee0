"""The gated delta rule on the GPU against its definition in 64 bits (tests/delta_reference.py): lengths around the chunk
of 32 tokens and around where the recurrence hands over to chunks, every element type, head dimension and layout, masks,
states, decays and keys where it can go wrong."""
import pytest
import torch

from delta_reference import DTYPES, check, inputs, reference

pytestmark = pytest.mark.gpu

NAMES = ("dQ", "dK", "dV", "dg", "dbeta")


def lay(t, layout):
    """[B,H,N,...] as the layout has it, contiguous, on the GPU."""
    if t is None:
        return None
    return (t if layout == "bhnd" else t.transpose(1, 2)).contiguous().cuda()


def back(t, layout):
    return t if layout == "bhnd" else t.transpose(1, 2)


def forward(x, layout="bhnd", scale=1.0, kept=False, states=True, **kw):
    from paper_2602_06935_amd import binding
    q, k, v, g, b = (lay(x[n], layout) for n in ("q", "k", "v", "g", "beta"))
    m = None if x["mask"] is None else x["mask"].cuda()
    S0 = None if x["S0"] is None else x["S0"].cuda()
    B, H, N, d = x["q"].shape
    S1 = torch.full((B, H, d, d), 7.0, device="cuda") if states else None
    held = binding.cotten_delta_kept(q, layout=layout) if kept else None
    O = binding.cotten_delta_fwd(q, k, v, g, b, m, scale=scale, layout=layout, initial_state=S0, final_state=S1, kept=held, **kw)
    torch.cuda.synchronize()
    return back(O, layout), S1, held


def backward(x, layout="bhnd", scale=1.0, kept=None, **kw):
    from paper_2602_06935_amd import binding
    q, k, v, g, b, dO = (lay(x[n], layout) for n in ("q", "k", "v", "g", "beta", "dO"))
    m = None if x["mask"] is None else x["mask"].cuda()
    S0, dS1 = (None if x[n] is None else x[n].cuda() for n in ("S0", "dS1"))
    B, H, N, d = x["q"].shape
    dS0 = torch.full((B, H, d, d), 7.0, device="cuda")
    got = binding.cotten_delta_bwd(q, k, v, g, b, m, dO, scale=scale, layout=layout, initial_state=S0, dfinal_state=dS1,
                                   dinitial_state=dS0, kept=kept, **kw)
    torch.cuda.synchronize()
    return dict(zip(NAMES, (back(t, layout) for t in got)), dS0=dS0)


def both(x, layout="bhnd", scale=1.0, eps=1e-6, kept=True):
    ref = reference(x, scale=scale, eps=eps)
    O, S1, held = forward(x, layout, scale, kept, eps=eps)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])
    got = backward(x, layout, scale, held, eps=eps)
    for n in NAMES + ("dS0",):
        check(n, got[n], ref[n])
    return O, S1, got


@pytest.mark.parametrize("N", [1, 2, 8, 9, 31, 32, 33, 64, 65, 97, 200])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_lengths(dtype, N):
    both(inputs(2, 2, N, 64, DTYPES[dtype], seed=N))


@pytest.mark.parametrize("N", [1, 7, 8])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_few_tokens(dtype, d, N):
    """The recurrence (no `kept` asked for), with states and a mask."""
    x = inputs(3, 2, N, d, DTYPES[dtype], seed=d + N, mask="holes", states=True)
    ref = reference(x, scale=0.5, grads=False)
    O, S1, _ = forward(x, scale=0.5)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_widths_masks_states(dtype, d, layout):
    both(inputs(3, 3, 75, d, DTYPES[dtype], seed=d, mask="holes", states=True), layout, scale=0.37)


@pytest.mark.parametrize("mask", ["left", "holes", "empty"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_rows_may_hold_anything(dtype, mask):
    x = inputs(4, 2, 70, 32, DTYPES[dtype], seed=5, mask=mask, states=True)
    dead = x["mask"] == 0
    for n, bad in (("k", float("nan")), ("v", float("inf")), ("g", float("nan")), ("beta", -float("inf"))):
        t = x[n].transpose(1, 2)          # [B,N,H,...]
        t[dead] = bad
        x[n] = t.transpose(1, 2).contiguous()
    O, S1, got = both(x)
    for n in ("dK", "dV", "dg", "dbeta"):
        assert (got[n].transpose(1, 2)[dead.cuda()] == 0).all(), n
    if mask == "empty":   # a sequence without a token: its state passes through, bit for bit
        assert torch.equal(S1[-1].cpu(), x["S0"][-1])


def test_masked_short_calls_may_hold_anything():
    x = inputs(4, 2, 5, 32, torch.bfloat16, seed=6, mask="empty", states=True)
    dead = x["mask"] == 0
    for n, bad in (("k", float("nan")), ("v", float("inf")), ("g", float("nan")), ("beta", float("nan"))):
        t = x[n].transpose(1, 2)
        t[dead] = bad
        x[n] = t.transpose(1, 2).contiguous()
    ref = reference(x, grads=False)
    O, S1, _ = forward(x)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])
    assert torch.equal(S1[-1].cpu(), x["S0"][-1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_of_every_size(dtype):
    """No decay, next to none, and a state emptied in the middle of a chunk (g = -60, -1000 and -inf), after which the
    weak decays still count."""
    x = inputs(2, 2, 100, 32, DTYPES[dtype], seed=7, states=True)
    x["g"][0] = 0.0
    x["g"][1, 0] *= 1e-5
    for t, g in ((10, -60.0), (43, -1000.0), (70, -float("inf"))):
        x["g"][1, :, t] = g
    ref = reference(x)
    ref["dg"] = torch.nan_to_num(ref["dg"], nan=0.0)     # (0 times -inf in the reference's own chain rule)
    O, S1, held = forward(x, kept=True)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])
    got = backward(x, kept=held)
    for n in NAMES + ("dS0",):
        check(n, got[n], ref[n])


def test_growing_states():
    x = inputs(1, 2, 64, 32, torch.float32, seed=8, states=True)
    x["g"] = -x["g"] * 0.2
    both(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_keys(dtype):
    """The same item again and again, beta = 1 and beta = 0: powers of the coupling matrix would grow to thousands."""
    x = inputs(2, 2, 96, 64, DTYPES[dtype], seed=9)
    x["k"][0] = x["k"][0, :, :1]
    x["beta"][0] = 1.0
    x["g"][0] = 0.0
    x["k"][1, :, 1::2] = x["k"][1, :, 0::2]
    x["beta"][1, :, ::3] = 0.0
    both(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_of_unusual_size(dtype):
    x = inputs(1, 2, 70, 64, DTYPES[dtype], seed=10)
    for n in ("q", "k"):
        x[n][0, :, 3::7] *= 1e-4
        x[n][0, :, 5::11] *= 0.0
        x[n][0, :, 1::9] *= 300.0
    both(x)


def test_eps_zero_with_masked_rows():
    x = inputs(2, 2, 40, 32, torch.float32, seed=11, mask="left", states=True)
    both(x, eps=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_without_kept_gives_the_same_bits(dtype):
    x = inputs(2, 3, 130, 64, DTYPES[dtype], seed=12, mask="left", states=True)
    _, _, held = forward(x, kept=True)
    first, again, alone = backward(x, kept=held), backward(x, kept=held), backward(x)
    for n in first:
        assert torch.equal(first[n], again[n]) and torch.equal(first[n], alone[n]), n


@pytest.mark.parametrize("cut", [1, 32, 50, 90])
def test_a_history_in_two_parts(cut):
    """The state that leaves the first part continues the second."""
    x = inputs(2, 2, 100, 64, torch.bfloat16, seed=13, mask="left")
    ref = reference(x, grads=False)
    parts = [{n: (t if n in ("S0", "dS1", "mask") else t[:, :, a:b].contiguous()) for n, t in x.items()}
             for a, b in ((0, cut), (cut, 100))]
    parts[0]["mask"], parts[1]["mask"] = x["mask"][:, :cut].contiguous(), x["mask"][:, cut:].contiguous()
    O0, S, _ = forward(parts[0])
    parts[1]["S0"] = S.cpu()
    O1, S, _ = forward(parts[1])
    check("O", torch.cat([O0, O1], 2), ref["O"])
    check("S1", S, ref["S1"])


def test_server_steps_in_place():
    from paper_2602_06935_amd import binding
    x = inputs(5, 2, 12, 64, torch.bfloat16, seed=14)
    ref = reference(x, grads=False)
    S = torch.zeros(5, 2, 64, 64, device="cuda")
    for t in range(12):
        q, k, v, g, b = (x[n][:, :, t:t + 1].contiguous().cuda() for n in ("q", "k", "v", "g", "beta"))
        O = binding.cotten_delta_fwd(q, k, v, g, b, None, initial_state=S, final_state=S)
        check("O", O, ref["O"][:, :, t:t + 1])
    check("S", S, ref["S1"])


def test_many_slices():
    """More workgroups than run at a time; the same sequence in every slice gives the same bits."""
    x = inputs(1, 1, 45, 32, torch.float32, seed=15, states=True)
    ref = reference(x)
    many = {n: (t if t is None else t.expand(700, 3, *t.shape[2:]).contiguous()) for n, t in x.items()}
    O, S1, held = forward(many, kept=True)
    got = backward(many, kept=held)
    for n, t in dict(got, O=O, S1=S1).items():
        assert torch.equal(t, t[:1, :1].expand_as(t)), n
        check(n, t[:1, :1], ref[n])


@pytest.mark.parametrize("slices", [600, 1200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_around_the_recurrence_of_many_slices(dtype, slices):
    """Both sides of the numbers of tokens up to which calls of many slices run as a recurrence."""
    for N in (8, 9, 10, 11, 16, 17):
        x = inputs(2, 1, N, 16, DTYPES[dtype], seed=N, states=True)
        ref = reference(x, grads=False)
        many = {n: (t if t is None else t.repeat(slices // 2, *[1] * (t.dim() - 1))) for n, t in x.items()}
        O, S1, _ = forward(many)
        check("O", O[:2], ref["O"])
        check("S1", S1[-2:], ref["S1"])
        assert torch.equal(O, O[:2].repeat(slices // 2, 1, 1, 1)) and torch.equal(S1, S1[:2].repeat(slices // 2, 1, 1, 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_history(dtype):
    both(inputs(1, 2, 1501, 32, DTYPES[dtype], seed=16, mask="left", states=True), "bnhd")


@pytest.mark.parametrize("N", [513, 1024, 1500])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_segments(dtype, d, N):
    """Few long sequences are cut into segments that run side by side."""
    x = inputs(1, 2, N, d, DTYPES[dtype], seed=N + d, mask="holes" if N == 1500 else None, states=True)
    if x["mask"] is not None:
        x["mask"][:] = (torch.rand(N, generator=torch.Generator().manual_seed(1)) < 0.7).to(torch.uint8)
    O, S1, _ = both(x, "bnhd" if N == 1024 else "bhnd", scale=0.5)
    if N != 1024:    # without what the backward needs, the same bits
        O2, S2, _ = forward(x, scale=0.5)
        assert torch.equal(O, O2) and torch.equal(S1, S2)


def test_segments_without_states():
    both(inputs(2, 1, 700, 32, torch.bfloat16, seed=21, mask="left"))


@pytest.mark.parametrize("kept", [False, True])
def test_segments_replace_a_state_in_place(kept):
    """The first segment reads the state that the last one writes."""
    from paper_2602_06935_amd import binding
    x = inputs(2, 2, 1500, 64, torch.bfloat16, seed=31, states=True)
    O, S1, _ = forward(x, kept=kept)
    q, k, v, g, b, S = (x[n].cuda() for n in ("q", "k", "v", "g", "beta", "S0"))
    held = binding.cotten_delta_kept(q) if kept else None
    for again in range(2):
        S.copy_(x["S0"])
        got = binding.cotten_delta_fwd(q, k, v, g, b, None, initial_state=S, final_state=S, kept=held)
        assert torch.equal(got, O) and torch.equal(S, S1)


def test_segments_backward_without_kept_gives_the_same_bits():
    x = inputs(1, 3, 900, 64, torch.bfloat16, seed=22, mask="left", states=True)
    _, _, held = forward(x, kept=True)
    first, alone = backward(x, kept=held), backward(x)
    for n in first:
        assert torch.equal(first[n], alone[n]), n


def test_gradient_against_differences():
    x = inputs(1, 2, 50, 32, torch.float32, seed=17, mask="left", states=True)
    _, _, held = forward(x, kept=True)
    got = backward(x, kept=held)

    def loss(y):
        O, S1, _ = forward(y)
        return (O.cpu().double() * x["dO"].double()).sum() + (S1.cpu().double() * x["dS1"].double()).sum()

    gen = torch.Generator().manual_seed(1)
    for n, grad in (("q", "dQ"), ("k", "dK"), ("v", "dV"), ("g", "dg"), ("beta", "dbeta"), ("S0", "dS0")):
        step = torch.randn(x[n].shape, generator=gen)
        h = 1e-3
        up, down = (dict(x, **{n: x[n] + s * h * step}) for s in (1.0, -1.0))
        slope = ((loss(up) - loss(down)) / (2 * h)).item()
        along = (got[grad].cpu().double() * step.double()).sum().item()
        # rounding of the two losses (a few hundred terms of size one, 1e-5 of each) over 2 h, and h^2 of curvature
        size = got[grad].cpu().double().norm().item()
        assert abs(slope - along) <= 2e-2 * size + 1e-2, (n, slope, along)


def test_another_stream_and_capture():
    """Captured with its backward and replayed among the program's own eager calls, on a side stream."""
    from paper_2602_06935_amd import binding
    for dtype, N in ((torch.bfloat16, 100), (torch.float32, 3)):
        x = inputs(2, 2, N, 64, dtype, seed=18, mask="left", states=True)
        q, k, v, g, b, dO, m, S0, dS1 = (x[n].cuda() for n in ("q", "k", "v", "g", "beta", "dO", "mask", "S0", "dS1"))
        S1, dS0 = torch.empty_like(S0), torch.empty_like(S0)
        held = binding.cotten_delta_kept(q)
        need = binding.cotten_delta_workspace_bytes(2, 2, N, 64, binding._dtype_code(q), True, True)
        space = torch.empty(need, dtype=torch.uint8, device="cuda")

        def calls():
            O = binding.cotten_delta_fwd(q, k, v, g, b, m, initial_state=S0, final_state=S1, kept=held)
            grads = binding.cotten_delta_bwd(q, k, v, g, b, m, dO, dfinal_state=dS1, dinitial_state=dS0, kept=held, workspace=space)
            short = binding.cotten_delta_fwd(q[:, :, :2].contiguous(), k[:, :, :2].contiguous(), v[:, :, :2].contiguous(),
                                             g[:, :, :2].contiguous(), b[:, :, :2].contiguous(), None)
            return (O, *grads, short)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = [t.clone() for t in calls()] + [S1.clone(), dS0.clone()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = calls()
        for _ in range(3):
            for t in (*out, S1, dS0):
                t.fill_(3.0)
            held.fill_(255)
            space.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, r) for p, r in zip((*out, S1, dS0), eager))
            again = [t.clone() for t in calls()]
            torch.cuda.synchronize()
            assert all(torch.equal(p, r) for p, r in zip(again, eager))


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_differentiable_function(layout):
    """Gradients through autograd, with the final state used, unused and not asked for."""
    from paper_2602_06935_amd.autograd import gated_delta_attention
    x = inputs(2, 2, 45, 32, torch.float32, seed=30, mask="left", states=True)
    names = ("q", "k", "v", "g", "beta")
    for with_state, use_state in ((True, True), (True, False), (False, False)):
        ref = reference(dict(x, dS1=x["dS1"] if use_state else None), scale=0.7)
        leaves = [lay(x[n], layout).requires_grad_() for n in names] + [x["S0"].cuda().requires_grad_()]
        got = gated_delta_attention(*leaves[:5], x["mask"].cuda(), scale=0.7, initial_state=leaves[5], return_state=with_state, layout=layout)
        outputs = got if use_state else (got[0] if with_state else got,)
        upstream = (lay(x["dO"], layout),) + ((x["dS1"].cuda(),) if use_state else ())
        grads = torch.autograd.grad(outputs, leaves, upstream)
        check("O", back(outputs[0], layout), ref["O"])
        for n, t in zip(NAMES, grads):
            check(n, back(t, layout), ref[n])
        check("dS0", grads[5], ref["dS0"])
    with torch.no_grad():
        O, S1 = gated_delta_attention(*leaves[:5], x["mask"].cuda(), scale=0.7, initial_state=leaves[5], return_state=True, layout=layout)
    check("S1", S1, ref["S1"])
