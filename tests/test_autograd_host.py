"""What the differentiable functions do around the library's calls, with stand-ins for these on the CPU."""
import pytest
import torch

from paper_2602_06935_amd import autograd, binding


@pytest.fixture
def stand_ins(monkeypatch):
    """Forward and backward calls that compute nothing, but return tensors of the right shapes; what backwards were given."""
    given = {}

    def delta_backward(prm, dims, Q, K, V, g, beta, mask, dO, initial_state, dfinal_state, dinitial_state, kept):
        given.update(dO=dO, dfinal_state=dfinal_state)
        return tuple(torch.ones_like(t) for t in (Q, K, V, g, beta))

    def attention_backward(Q, K, V, mask, dO, **kw):
        given.update(dO=dO)
        return tuple(torch.ones_like(Q) for _ in range(3))

    monkeypatch.setattr(binding, "cotten_attn_fwd", lambda Q, *a, **kw: Q.detach() + 1.0)
    monkeypatch.setattr(binding, "cotten_attn_bwd", attention_backward)
    monkeypatch.setattr(binding, "cotten_delta_kept", lambda Q, **kw: torch.zeros(8))
    monkeypatch.setattr(binding, "cotten_delta_fwd", lambda Q, *a, **kw: Q.detach() + 1.0)
    monkeypatch.setattr(binding, "_delta_backward_of", delta_backward)
    monkeypatch.setattr(binding, "cotten_embed_fwd", lambda ids, W, *a, **kw: W.detach().new_ones(*ids.shape, W.shape[1]))
    monkeypatch.setattr(binding, "_embed_backward_of",
                        lambda prm, ids, dE, W_shape, P_shape, *a: (dE.new_ones(W_shape), None if P_shape is None else dE.new_ones(P_shape)))
    return given


def leaves(*shapes):
    return [torch.randn(s).requires_grad_() for s in shapes]


def outputs():
    q, k, v, g, beta = leaves(*[(1, 1, 4, 16)] * 3, *[(1, 1, 4)] * 2)
    yield "attention", q, autograd.cosine_attention(q, k, v)
    yield "delta", q, autograd.gated_delta_attention(q, k, v, g, beta)
    W, P = leaves((5, 8), (4, 8))
    yield "embedding", W, autograd.item_embedding(torch.zeros(2, 3, dtype=torch.int64), W, P)


def test_second_derivatives_raise(stand_ins):
    """A penalty on the gradients would lose its term: the kernels' gradients do not say what they depend on."""
    for name, x, y in outputs():
        first, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(y.sum() + first.square().sum(), x)
            pytest.fail(name)
        first, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            (y.sum() + first.square().sum()).backward()
            pytest.fail(name)


def test_second_derivatives_raise_where_the_upstream_gradient_is_constant(stand_ins):
    """... but not the inputs that it meets."""
    for name, x, y in outputs():
        if name == "embedding":     # linear: its gradient depends on the upstream gradient alone
            continue
        first, = torch.autograd.grad(y.sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(y.sum() + first.square().sum(), x)
            pytest.fail(name)


def test_graphs_of_first_derivatives_are_allowed(stand_ins):
    """What does not go on through the kernels' gradients does not raise, and these are what they are without a graph."""
    for name, x, y in outputs():
        plain, = torch.autograd.grad((y * y).sum(), x, retain_graph=True)
        first, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        assert torch.equal(first, plain), name
        torch.autograd.grad(y.sum() + first.detach().sum(), x)


def test_upstream_gradients_may_begin_anywhere(stand_ins):
    """The gradient of a part behind an odd one is a contiguous view off the boundaries that the library asks for."""
    q, k, v, g, beta = leaves(*[(1, 1, 4, 16)] * 3, *[(1, 1, 4)] * 2)
    O, S = autograd.gated_delta_attention(q, k, v, g, beta, return_state=True)
    for outputs, names in (((O, S), ("dO", "dfinal_state")), ((autograd.cosine_attention(q, k, v),), ("dO",))):
        for out, name in zip(outputs, names):
            factor = torch.randn(3 + out.numel())
            stand_ins.clear()
            torch.autograd.grad((torch.cat([q.flatten()[:3], out.flatten()]) * factor).sum(), q, retain_graph=True)
            got = stand_ins[name]
            assert got.data_ptr() % 16 == 0 and got.is_contiguous()
            assert torch.equal(got.flatten(), factor[3:])


def test_gradients_that_nobody_wants_are_not_computed(monkeypatch, stand_ins):
    """Positions that are trained over a table that is not: the table's gradient is a sort and a write of all of it."""
    wanted = []

    def backward(prm, ids, dE, W_shape, P_shape, of_table=True):
        wanted.append((of_table, P_shape is not None))
        return dE.new_ones(W_shape) if of_table else None, None if P_shape is None else dE.new_ones(P_shape)

    monkeypatch.setattr(binding, "_embed_backward_of", backward)
    ids = torch.zeros(2, 3, dtype=torch.int64)
    for of_W, of_P in ((True, True), (True, False), (False, True)):
        W, P = torch.randn(5, 8, requires_grad=of_W), torch.randn(4, 8, requires_grad=of_P)
        autograd.item_embedding(ids, W, P).sum().backward()
        assert wanted.pop() == (of_W, of_P)
        assert (W.grad is not None, P.grad is not None) == (of_W, of_P)


def test_nothing_is_kept_for_a_backward_that_cannot_come(monkeypatch, stand_ins):
    """Under no_grad tensors still say that they want gradients; the states of all chunks are not written for that."""
    kept = []
    monkeypatch.setattr(binding, "cotten_delta_fwd", lambda Q, *a, **kw: kept.append(kw["kept"]) or Q.detach() + 1.0)
    q, k, v, g, beta = leaves(*[(1, 1, 4, 16)] * 3, *[(1, 1, 4)] * 2)
    autograd.gated_delta_attention(q, k, v, g, beta)
    assert kept.pop() is not None
    with torch.no_grad():
        autograd.gated_delta_attention(q, k, v, g, beta)
    assert kept.pop() is None
    autograd.gated_delta_attention(*(t.detach() for t in (q, k, v, g, beta)))
    assert kept.pop() is None
