"""The operators together, as the example's model uses them: embedding, dropout, decay attention and seam trained, the same served
item by item, and slates by beam search with the states behind their beams."""
import math
import os
import sys

import pytest
import torch

from seam_reference import factors

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def example(monkeypatch):
    monkeypatch.syspath_prepend(os.path.join(ROOT, "examples"))
    import next_item
    return next_item


def plain(model, ids, p=0.0, call=0):
    """The model's scores from the operators' definitions, in 64 bits on the CPU; and its parameters there."""
    w = {n: t.detach().cpu().double().requires_grad_() for n, t in model.named_parameters()}
    B, N = ids.shape
    D, H = w["W"].shape[1], model.heads
    live = (ids != 0)
    E = torch.where(live[..., None], model.scale * w["W"][ids.long()], 0.0) + w["P"][:N]
    drop = [1.0, 1.0]
    if p > 0:
        drop = [factors(E.numel(), p, model.seed, 2 * call + i).reshape(E.shape) for i in range(2)]
    E = E * drop[0]
    q, k, v = (t.reshape(B, N, H, D // H) for t in (E @ w["qkv.weight"].t() + w["qkv.bias"]).chunk(3, -1))
    q, k = (t / (t.square().sum(-1, keepdim=True) + 1e-6).sqrt() for t in (q, k))
    a = torch.exp(-torch.nn.functional.softplus(w["forget"]))
    S, o = torch.zeros(B, H, D // H, D // H, dtype=torch.float64), []
    for t in range(N):
        S = torch.where(live[:, t, None, None, None], a[None, :, None, None] * S + k[:, t, :, :, None] * v[:, t, :, None, :], S)
        o.append((q[:, t, :, :, None] * S).sum(-2))
    F = torch.stack(o, 1).flatten(2) @ w["out.weight"].t() + w["out.bias"]
    unit = lambda x: x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()               # noqa: E731
    X = E + w["gate"] * (unit(F) * w["after"] * drop[1])
    return (unit(X) * w["before"]) @ w["W"].t() / model.scale, w


def make(example, items, longest, p=0.0, width=32, seed=3):
    torch.manual_seed(seed)
    return example.DecayItem(items, longest, width=width, heads=2, dtype=torch.float32, p=p).cuda()


@pytest.mark.parametrize("p", [0.0, 0.2])
def test_gradients_of_the_whole_model(example, p):
    """Every parameter's, against differentiating the definitions: each operator is within 1e-5 of its own, five of them and three
    torch products in 32 bits follow each other, and a gradient passes them twice."""
    model = make(example, 60, 40, p=p)
    gen = torch.Generator().manual_seed(5)
    ids = torch.randint(1, 60, (6, 37), generator=gen)
    ids[torch.arange(37)[None, :] < torch.randint(0, 30, (6, 1), generator=gen)] = 0
    up = torch.randn(6, 37, 60, generator=gen)
    scores = model(ids.cuda())
    want, w = plain(model, ids, p)
    assert (scores.detach().cpu().double() - want).norm() <= 1e-4 * want.norm()
    names = [n for n, _ in model.named_parameters()]
    got = torch.autograd.grad(scores, [t for _, t in model.named_parameters()], up.cuda())
    ref = torch.autograd.grad(want, [w[n] for n in names], up.double())
    for n, a, b in zip(names, got, ref):
        assert (a.cpu().double() - b).norm() <= 1e-4 * b.norm(), n


def test_calls_draw_anew(example):
    model = make(example, 30, 20, p=0.3)
    ids = torch.randint(1, 30, (3, 20), device="cuda")
    with torch.no_grad():
        first, second = model(ids), model(ids)
        assert not torch.equal(first, second)
        want, _ = plain(model, ids.cpu(), 0.3, call=1)
    assert (second.cpu().double() - want).norm() <= 1e-4 * want.norm()


@pytest.mark.parametrize("mixer", ["decay", "delta"])
def test_slates_are_the_best_there_are(example, mixer):
    """As many beams as items: nothing is lost after the first, so two items' slates are the best of all pairs, which are scored one by
    one by whole histories."""
    V, N, B = 12, 15, 3
    torch.manual_seed(4)
    model = make(example, V, N + 2) if mixer == "decay" else example.NextItem(V, N + 2, width=32, heads=2, dtype=torch.float32).cuda()
    model.eval()
    model.W.data.mul_(6.0)                                # (scores further apart than their roundings)
    gen = torch.Generator().manual_seed(6)
    ids = torch.randint(1, V, (B, N), generator=gen)
    ids[0, :7] = 0
    state = torch.zeros(B, 2, 16, 16, device="cuda")
    for t in range(N):
        scores = model.take_in(ids[:, t:t + 1].contiguous().cuda(), state, t)
    items, total = example.slates(model, state, scores, N, V, 2)
    with torch.no_grad():
        pairs = torch.cartesian_prod(torch.arange(1, V), torch.arange(1, V))
        for b in range(B):
            whole = torch.cat([ids[b].expand(len(pairs), N), pairs[:, :1]], 1)
            logits = model(whole.cuda())[:, -2:].double().cpu()
            logits[..., 0] = -math.inf
            logp = torch.log_softmax(logits, -1)
            of_pair = logp[:, 0].gather(1, pairs[:, :1])[:, 0] + logp[:, 1].gather(1, pairs[:, 1:])[:, 0]
            best, at = of_pair.sort(descending=True)
            # two scores of 32 bits of the model each way, of size 10 at most
            assert (total[b].cpu().double() - best[:V]).abs().max() < 1e-4
            for k in range(V):
                here = (pairs == items[b, k].cpu()).all(1).nonzero().item()
                assert abs(of_pair[here].item() - best[k].item()) < 1e-4


@pytest.mark.parametrize("mixer,p", [("decay", "0.1"), ("delta", "0")])
@pytest.mark.parametrize("dtype,bar", [("f32", 1e-4), ("bf16", 4e-2)])
def test_example_runs(example, monkeypatch, dtype, bar, mixer, p):
    """Bars: the outputs of the layer differ by roundings of their type (2^-8 in bf16), which the projections and the
    products with the item table carry on, a few of them one behind the other."""
    monkeypatch.setattr(sys, "argv", ["next_item.py", "--steps", "4", "--dtype", dtype, "--mixer", mixer, "--dropout", p, "--slates", "4",
                                      "--items", "80", "--users", "32"])
    losses, far = example.main()
    assert all(math.isfinite(x) for x in losses) and far < bar


def test_a_captured_training_pass():
    """Forward and backward of mixer, seam and dropout in one graph; replays follow the inputs and draw anew."""
    from paper_2602_06935_amd import autograd
    gen = torch.Generator().manual_seed(5)
    draw = lambda *shape: torch.randn(*shape, generator=gen).to("cuda", torch.bfloat16)        # noqa: E731
    B, N, H, d = 3, 300, 2, 64
    q, k, v = (draw(B, N, H, d).requires_grad_() for _ in range(3))
    X = draw(B, N, H * d).requires_grad_()
    g = torch.full((H,), -0.05, device="cuda").requires_grad_()
    post, after = (draw(H * d).requires_grad_() for _ in range(2))
    mask = (torch.rand(B, N, generator=gen) < 0.8).to(torch.uint8).cuda()
    up = [draw(B, N, H * d) for _ in range(2)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    leaves = (q, k, v, g, X, post, after)

    def run():
        O = autograd.decay_attention(q, k, v, g, mask, layout="bnhd")
        Y, h = autograd.residual_norm(X, O.reshape(B, N, H * d), post_weight=post, next_weight=after, p=0.1, seed=2, step=step)
        return (Y, *torch.autograd.grad((Y, autograd.dropout(h, 0.3, seed=2, offset=1 << 40, step=step)), leaves, up))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = [t.detach() for t in run()]
    for i in range(4):
        with torch.no_grad():
            v.mul_(-0.9)
            step.fill_(i)
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
