"""Embedding of item ids and its gradient on the GPU against sums in 64 bits.

Bounds: E is one fused multiply-add and a rounding, at most eps / 2 of scale * W + P's terms; a gradient is a fp32 sum of m
terms in groups of sixteen (at most m / 16 + 16 roundings of 2^-24, in the mean far fewer: sqrt of that times two of the
sum of squares' root) and one rounding to its type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make(B, N, D, V, dtype, seed=0, positions=True, skew=True, wide=True):
    gen = torch.Generator().manual_seed(seed)
    u = torch.rand(B, N, generator=gen)
    ids = torch.exp(u * math.log(V)).long().clamp(0, V - 1) if skew else torch.randint(0, V, (B, N), generator=gen)
    W = torch.randn(V, D, generator=gen).to(dtype)
    P = torch.randn(N + 5, D, generator=gen).to(dtype) if positions else None
    dE = torch.randn(B, N, D, generator=gen).to(dtype)
    return ids if wide else ids.int(), W, P, dE


def reference(ids, W, P, dE, scale, padding, offset):
    V, D = W.shape
    B, N = ids.shape
    ids = ids.long()
    live = (ids >= 0) & (ids < V) & (ids != (-1 if padding is None else padding))
    rows = torch.where(live, ids, 0)
    E = torch.where(live[..., None], scale * W.double()[rows], torch.zeros((), dtype=torch.float64))
    if P is not None:
        E = E + P.double()[offset:offset + N]
    dW = torch.zeros(V, D, dtype=torch.float64)
    dW.index_add_(0, rows[live], dE.double()[live])
    many = torch.zeros(V, dtype=torch.float64).index_add_(0, rows[live], torch.ones(int(live.sum()), dtype=torch.float64))
    squares = torch.zeros(V, D, dtype=torch.float64).index_add_(0, rows[live], dE.double()[live].square())
    dP = None
    if P is not None:
        dP = torch.zeros(P.shape, dtype=torch.float64)
        dP[offset:offset + N] = dE.double().sum(0)
    return E, dW * scale, dP, many, squares.sqrt() * abs(scale)


def run_and_check(ids, W, P, dE, scale=1.0, padding=None, offset=0, **kw):
    from paper_2602_06935_amd import binding
    E, dW, dP, many, size = reference(ids, W, P, dE, scale, padding, offset)
    i, w, g = ids.cuda(), W.cuda(), dE.cuda()
    p = None if P is None else P.cuda()
    opts = dict(scale=scale, padding_idx=padding, position_offset=offset)
    got = binding.cotten_embed_fwd(i, w, p, **opts)
    torch.cuda.synchronize()
    half = torch.finfo(W.dtype).eps / 2
    terms = E.abs() + (0 if P is None else 2 * P.double()[offset:offset + ids.shape[1]].abs())
    assert ((got.cpu().double() - E).abs() <= (half + 2.0 ** -23) * terms + 1e-30 + (6e-8 if W.dtype is torch.float16 else 0)).all()
    gp = None if P is None else torch.full_like(p, 7.0)
    gw = binding.cotten_embed_bwd(i, g, W.shape[0], torch.full_like(w, 7.0), gp, **opts, **kw)
    again = binding.cotten_embed_bwd(i, g, W.shape[0], **opts)
    torch.cuda.synchronize()
    assert torch.equal(gw, again)
    slack = 2.0 ** -24 * (many / 16 + 32)[:, None] * size + (6e-8 if W.dtype is torch.float16 else 1e-30)
    off = (gw.cpu().double() - dW).abs() - half * dW.abs() * 1.01
    assert (off <= slack).all(), (off - slack).max()
    assert (gw.cpu()[many == 0] == 0).all()
    if P is not None:
        B = ids.shape[0]
        slack = 2.0 ** -24 * (B / 4 + 32) * math.sqrt(B) * 4 + (6e-8 if W.dtype is torch.float16 else 0)
        assert ((gp.cpu().double() - dP).abs() <= half * dP.abs() * 1.01 + slack).all()
        assert (gp.cpu()[:offset] == 0).all() and (gp.cpu()[offset + ids.shape[1]:] == 0).all()
    return got, gw, gp


@pytest.mark.parametrize("D", [1, 3, 8, 17, 64, 99, 100, 128, 256, 300, 1030])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_widths(dtype, D):
    run_and_check(*make(7, 19, D, 40, DTYPES[dtype], seed=D), scale=math.sqrt(D), padding=0)


@pytest.mark.parametrize("B,N,V", [(1, 1, 1), (1, 1, 50), (3, 5, 2), (1, 16, 3), (1, 17, 3), (2, 16, 1), (13, 63, 1),
                                   (64, 128, 500), (16, 512, 7), (41, 200, 3700), (64, 129, 600), (100, 90, 120000),
                                   (60, 150, 511), (60, 150, 512), (60, 150, 262143), (60, 150, 262144), (60, 150, 300000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lists_of_tokens(dtype, B, N, V):
    """One token, units that end with a row and inside one, rows over many units, one workgroup's sort and many's (from
    8193 tokens on), one digit, two and three."""
    run_and_check(*make(B, N, 32, V, DTYPES[dtype], seed=V), padding=None if V < 3 else 2)


@pytest.mark.parametrize("skew", [True, False])
def test_many_tokens(skew):
    ids, W, P, dE = make(300, 200, 64, 5000, torch.float32, seed=3, skew=skew)
    ids[:, :40] = 7          # one item of every sixth token
    run_and_check(ids, W, P, dE, scale=8.0, padding=0, offset=3)


@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("B,N", [(6, 20), (100, 100)])
def test_tokens_without_a_row(B, N, wide):
    """Padding, negative ids and ids beyond the table: nothing is read or written for them."""
    ids, W, P, dE = make(B, N, 24, 30, torch.bfloat16, seed=4, wide=wide)
    ids[0] = 5
    ids[1, ::2] = -1
    ids[2] = 30
    ids[3, 1:] = 2 ** 31 - 1
    if wide:
        ids[4] = 2 ** 32 + 3
        ids[5] = -2 ** 40
    run_and_check(ids, W, P, dE, padding=5, scale=0.5)


@pytest.mark.parametrize("B,N,D", [(1, 300, 17), (2, 700, 64), (3, 40, 32), (64, 1, 64), (65, 1, 64), (200, 3, 99), (4097, 1, 256),
                                   (5000, 1, 3), (1100, 7, 300), (300, 30, 1030)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_positions_of_few_and_many_sequences(dtype, B, N, D):
    """Sums over the sequences in parts, in one, and over next to none."""
    ids, W, P, dE = make(B, N, D, 40, DTYPES[dtype], seed=B + N)
    run_and_check(ids, W, P, dE, offset=3)


@pytest.mark.parametrize("many", [17, 1024, 1025, 1040, 2063, 2064, 2065, 65552, 70000])
def test_rows_of_many_units(many):
    """One id takes 64 units of sixteen tokens, a few more or fewer, or thousands, between others."""
    ids, W, P, dE = make(1, many + 40, 8, 9, torch.float32, seed=many, positions=False)
    ids[:] = torch.arange(many + 40) % 9
    ids[ids == 4] = 5
    ids[0, 30:30 + many] = 4
    run_and_check(ids, W, None, dE)


@pytest.mark.parametrize("D", [1, 3, 8, 17, 64, 100, 300, 1030])
@pytest.mark.parametrize("tokens", [2047, 2048, 2049, 8192, 8193])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_and_many_tokens_of_every_width(dtype, tokens, D):
    """Up to 2048 and up to 8192 tokens go in one launch, more are sorted first."""
    ids, W, P, dE = make(1, tokens, D, 700, DTYPES[dtype], seed=tokens + D)
    run_and_check(ids, W, P, dE, scale=0.5, padding=3)


@pytest.mark.parametrize("V", [1, 2, 50, 511, 513, 3000, 120000])
@pytest.mark.parametrize("B,N", [(1, 1), (7, 9), (40, 51), (2048, 1)])
def test_few_tokens_of_tables_of_every_size(B, N, V):
    ids, W, P, dE = make(B, N, 32, V, torch.bfloat16, seed=V + N)
    run_and_check(ids, W, P, dE, offset=2)
    run_and_check(ids.int(), W, None, dE, scale=3.0)


@pytest.mark.parametrize("tokens", [2500, 9000])
@pytest.mark.parametrize("many", [15, 16, 17, 32, 1024, 1025, 1040, 2064])
def test_a_popular_id(many, tokens):
    ids, W, P, dE = make(1, tokens, 8, 9, torch.float32, seed=many, positions=False)
    ids[:] = torch.arange(tokens) % 9
    ids[ids == 4] = 5
    ids[0, 300:300 + many] = 4
    run_and_check(ids, W, None, dE)


def test_no_token_has_a_row():
    ids, W, P, dE = make(4, 50, 16, 9, torch.float32, seed=5)
    ids[:] = 0
    run_and_check(ids, W, P, dE, padding=0)
    run_and_check(ids, W, None, dE, padding=0)


def test_one_token_a_call_with_positions():
    ids, W, P, dE = make(33, 1, 64, 100, torch.float16, seed=6)
    for offset in range(6):
        run_and_check(ids, W, P, dE, offset=offset, scale=8.0)


def test_gradient_is_that_of_the_forward():
    from paper_2602_06935_amd.autograd import item_embedding
    ids, W, P, dE = make(5, 30, 32, 20, torch.float32, seed=7)
    w, p, i, g = W.cuda().requires_grad_(), P.cuda().requires_grad_(), ids.cuda(), dE.cuda()
    E = item_embedding(i, w, p, scale=3.0, padding_idx=1, position_offset=2)
    dw, dp = torch.autograd.grad(E, (w, p), g)
    gen = torch.Generator().manual_seed(8)
    for t, grad in ((W, dw), (P, dp)):      # E is linear in both: a difference is exact but for rounding
        step = torch.randn(t.shape, generator=gen)
        a, b = (item_embedding(i, *(x.cuda() for x in ((W + s * step, P) if t is W else (W, P + s * step))), scale=3.0,
                               padding_idx=1, position_offset=2).cpu().double() for s in (1.0, -1.0))
        slope = ((a - b) / 2 * dE.double()).sum().item()
        along = (grad.cpu().double() * step.double()).sum().item()
        assert abs(slope - along) <= 1e-4 * grad.cpu().double().norm().item() * math.sqrt(step.numel())


def test_gradient_that_begins_anywhere():
    """The gradient of a part of a concatenation is a view whose rows of 198 bytes begin off 16-byte boundaries."""
    from paper_2602_06935_amd.autograd import item_embedding
    ids, W, _, _ = make(3, 5, 99, 20, torch.float16, seed=9, positions=False)
    w, i = W.cuda().requires_grad_(), ids.cuda()
    g = torch.randn(6, 5, 99, generator=torch.Generator().manual_seed(10)).half()
    both = torch.cat([item_embedding(i, w), item_embedding(i, w, scale=2.0)])
    dw, = torch.autograd.grad(both, w, g.cuda())
    want = torch.zeros(20, 99, dtype=torch.float64)
    for part, scale in ((g[:3], 1.0), (g[3:], 2.0)):
        want.index_add_(0, ids.flatten(), part.double().flatten(0, 1), alpha=scale)
    # two gradients and their sum, each rounded once
    size = torch.zeros(20, 99, dtype=torch.float64).index_add_(0, ids.flatten(), (g[:3].double().abs() + 2 * g[3:].double().abs()).flatten(0, 1))
    assert ((dw.cpu().double() - want).abs() <= 2 * torch.finfo(torch.float16).eps / 2 * size + 1e-6).all()


def test_capture_and_another_stream():
    from paper_2602_06935_amd import binding
    for B, N in ((9, 40), (90, 110)):
        ids, W, P, dE = make(B, N, 64, 700, torch.bfloat16, seed=9)
        i, w, p, g = ids.cuda(), W.cuda(), P.cuda(), dE.cuda()
        dW, dP = torch.empty_like(w), torch.empty_like(p)
        space = torch.empty(binding.cotten_embed_workspace_bytes(B, N, 64, 700), dtype=torch.uint8, device="cuda")

        def calls():
            E = binding.cotten_embed_fwd(i, w, p, scale=8.0, padding_idx=0)
            binding.cotten_embed_bwd(i, g, 700, dW, dP, scale=8.0, padding_idx=0, workspace=space)
            return E, dW, dP

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            eager = [t.clone() for t in calls()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = calls()
        for _ in range(3):
            for t in out:
                t.fill_(3.0)
            space.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, eager))
            again = [t.clone() for t in calls()]
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(again, eager))
