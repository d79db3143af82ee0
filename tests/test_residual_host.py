"""Dropout and the seam on the host: the generator's published values, what the C calls refuse before any device work (the
pointers here are never followed), and what the bindings refuse."""
import ctypes

import pytest
import torch

from paper_2602_06935_amd import autograd, binding
from seam_reference import factors, philox


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def test_generator_of_the_reference():
    """Known answers of Philox4x32 with ten rounds, as its authors publish them."""
    assert philox([0] * 4, (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert philox([0xffffffff] * 4, (0xffffffff, 0xffffffff)) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    kept = (factors(1 << 16, 0.25, 5, 1) > 0).double().mean().item()
    assert abs(kept - 0.75) < 5 * (0.25 * 0.75 / (1 << 16)) ** 0.5


def dropout(lib, x=0x1000, y=0x2000, n=100, **kw):
    p = binding.CottenDropoutParams(0, 0.1, 1, 2, None)
    for k, v in kw.items():
        setattr(p, k, v)
    return lib.cotten_dropout(x, y, n, None, ctypes.byref(p))


def test_dropout_refusals(lib):
    assert lib.cotten_dropout(0x1000, 0x2000, 8, None, None) == -1
    assert dropout(lib, x=None) == -1 and dropout(lib, y=None) == -1
    assert dropout(lib, x=0x1008) == -5 and dropout(lib, y=0x2004) == -5 and dropout(lib, step=0x3004) == -5
    assert dropout(lib, n=0) == -2 and dropout(lib, n=1 << 40) == -2
    assert dropout(lib, dtype=3) == -4
    for p in (-0.1, 1.0, 1.5, float("nan"), 1 - 2.0 ** -18):
        assert dropout(lib, p=p) == -7, p


def params(**kw):
    p = binding.CottenResidualParams(dtype=0, norm=1, post_weight=0x10000, post_bias=0x11000, gate=0x12000, next_weight=0x13000,
                                     next_bias=0x14000, alpha=1.0, eps=-1.0, workspace=0x20000, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


FWD = (0x1000, 0x2000, 0x3000, 0x4000)
BWD = (0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000)


def forward(lib, ptrs=FWD, dims=(2, 3, 64), **kw):
    return lib.cotten_residual_fwd(*ptrs, *dims, None, ctypes.byref(params(**kw)))


def backward(lib, ptrs=BWD, dims=(2, 3, 64), grads=(0x7000, 0x7100, 0x7200, 0x7300, 0x7400), **kw):
    return lib.cotten_residual_bwd(*ptrs, *dims, None, ctypes.byref(params(**kw)),
                                   ctypes.byref(binding.CottenResidualGrads(*grads)))


@pytest.mark.parametrize("call,ptrs", [(forward, FWD), (backward, BWD)])
def test_seam_refusals(lib, call, ptrs):
    for i in range(len(ptrs)):
        assert call(lib, ptrs[:i] + (ptrs[i] + 8,) + ptrs[i + 1:]) == -5, i
        if call is forward or i not in (2, 3):
            assert call(lib, ptrs[:i] + (None,) + ptrs[i + 1:]) == -1, i
    for name in ("post_weight", "post_bias", "gate", "next_weight", "next_bias", "workspace"):
        assert call(lib, **{name: 0x10008}) == -5, name
    for dims in ((0, 3, 64), (2, 0, 64), (2, 3, 0), (2, 3, 8193), (1 << 16, 1 << 15, 64)):
        assert call(lib, dims=dims) == -2, dims
    assert call(lib, dtype=3) == -4
    assert call(lib, norm=2) == -7
    assert call(lib, post_weight=None) == -7                       # a bias without its weight
    for bad in (float("nan"), float("inf")):
        assert call(lib, alpha=bad) == -7 and call(lib, eps=bad) == -7
    assert call(lib, p=1.0) == -7 and call(lib, p=-0.5) == -7 and call(lib, p=float("nan")) == -7
    assert call(lib, step=0x30004) == -5


def test_seam_forward_refuses_half_a_norm(lib):
    assert forward(lib, next_weight=None, next_bias=None) == -1     # H without its norm
    assert forward(lib, FWD[:3] + (None,)) == -1


def test_seam_backward_refusals(lib):
    assert lib.cotten_residual_bwd(*BWD, 2, 3, 64, None, ctypes.byref(params()), None) == -1
    assert lib.cotten_residual_bwd(*BWD, 2, 3, 64, None, None, ctypes.byref(binding.CottenResidualGrads())) == -1
    assert backward(lib, BWD[:2] + (None, None) + BWD[4:]) == -1
    assert backward(lib, next_weight=None, next_bias=None) == -7
    assert backward(lib, grads=(0x7000, 0x7100, 0x7200, 0x7300, 0x7408)) == -5
    assert backward(lib, gate=None) == -7 and backward(lib, next_bias=None) == -7
    for per_sequence in (0, 1):
        need = binding.cotten_residual_workspace_bytes(2, 3, 64, bool(per_sequence))
        assert need > 0
        assert backward(lib, gate_per_sequence=per_sequence, workspace_bytes=need - 1) == -6
    assert backward(lib, workspace=None) == -6
    assert binding.cotten_residual_workspace_bytes(0, 1, 8) == 0 and binding.cotten_residual_workspace_bytes(1, 1, 20000) == 0


def test_bindings_refuse():
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_dropout(x, 0.1, seed=0)
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_residual_fwd(x, x)
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_residual_bwd(x, x, x, None)
    for p, seed, offset in ((1.0, 0, 0), (-0.1, 0, 0), (float("nan"), 0, 0), (0.1, -1, 0), (0.1, 2 ** 64, 0), (0.1, 0, -1), (0.1, 0, 2 ** 64)):
        with pytest.raises(ValueError):
            binding._check_generator(p, seed, offset, None, x.device)
    for step in (torch.zeros(1), torch.zeros(2, dtype=torch.int64)):
        with pytest.raises(ValueError, match="step"):
            binding._check_generator(0.1, 0, 0, step, x.device)


def test_second_derivatives_raise(monkeypatch):
    monkeypatch.setattr(binding, "cotten_dropout", lambda x, p, **kw: x.detach() * 2.0)
    monkeypatch.setattr(binding, "cotten_residual_fwd", lambda X, F, **kw: (X.detach() + F.detach(), X.detach() + 1.0))
    monkeypatch.setattr(binding, "_residual_backward_of", lambda call, X, F, *a: (torch.ones_like(X), torch.ones_like(F), *(None,) * 5))
    for run in (lambda x: autograd.dropout(x, 0.5, seed=1), lambda x: autograd.residual_norm(x, x * 2.0)[0]):
        x = torch.randn(2, 3, 8, requires_grad=True)
        y = run(x)
        first, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(y.sum() + first.square().sum(), x)


def test_step_may_not_change_before_the_backward(monkeypatch):
    monkeypatch.setattr(binding, "cotten_dropout", lambda x, p, **kw: x.detach() * 2.0)
    x, step = torch.randn(4, requires_grad=True), torch.zeros(1, dtype=torch.int64)
    y = autograd.dropout(x, 0.5, seed=1, step=step)
    step += 1
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()
