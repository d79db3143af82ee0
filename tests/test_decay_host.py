"""What the decay attention refuses on the host, before any device work (the pointers here are never followed), and what the
differentiable function does around the calls."""
import ctypes

import pytest
import torch

from paper_2602_06935_amd import autograd, binding


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def params(**kw):
    p = binding.CottenDecayParams(binding.COTTEN_F32, 0.0, -1.0, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


FWD = (0x1000, 0x2000, 0x3000, 0x4000, None, 0x5000)
BWD = (0x1000, 0x2000, 0x3000, 0x4000, None, 0x5000, 0x6000, 0x7000, 0x8000, 0x9000)


def forward(lib, ptrs=FWD, dims=(2, 2, 40, 32), **kw):
    return lib.cotten_decay_fwd(*ptrs, *dims, None, ctypes.byref(params(**kw)))


def backward(lib, ptrs=BWD, dims=(2, 2, 40, 32), **kw):
    return lib.cotten_decay_bwd(*ptrs, *dims, None, ctypes.byref(params(**kw)))


@pytest.mark.parametrize("call,ptrs", [(forward, FWD), (backward, BWD)])
def test_refusals(lib, call, ptrs):
    room = dict(workspace=0x100000, workspace_bytes=1 << 40)
    for i in range(len(ptrs)):
        if i == 4:
            continue
        if i != 9:      # (dg may be left out)
            assert call(lib, ptrs[:i] + (None,) + ptrs[i + 1:], **room) == -1, i
        assert call(lib, ptrs[:i] + (ptrs[i] + 2,) + ptrs[i + 1:], **room) == -5, i
    fn = lib.cotten_decay_fwd if call is forward else lib.cotten_decay_bwd
    assert fn(*ptrs, 2, 2, 40, 32, None, None) == -1
    for dims in ((0, 2, 40, 32), (2, 0, 40, 32), (2, 2, 0, 32), (2, 2, -1, 32), (1 << 11, 1 << 10, 40, 32), (1, 1, 1 << 25, 16),
                 (1, 1, 1 << 24, 32)):
        assert call(lib, ptrs, dims, **room) == -2, dims
    for N in (1, 2, 16):
        assert call(lib, ptrs, (1, 1 << 20, N, 64), layout=1, **room) == -2, N      # 32 rows of 2^28 bytes
    for d in (0, 8, 48, 96, 256):
        assert call(lib, ptrs, (2, 2, 40, d), **room) == -3
    assert call(lib, ptrs, dtype=3, **room) == -4
    assert call(lib, ptrs, layout=2, **room) == -2
    for bad in (float("nan"), float("inf")):
        assert call(lib, ptrs, scale=bad, **room) == -7
        assert call(lib, ptrs, eps=bad, **room) == -7
    for name in ("initial_state", "final_state", "dfinal_state", "dinitial_state", "workspace"):
        assert call(lib, ptrs, **dict(room, **{name: 0x10004})) == -5, name


def test_workspaces(lib):
    size = binding.cotten_decay_workspace_bytes
    long = (1, 2, 2000, 64)
    assert size(2, 2, 40, 32, 0, False) == 0 and size(*long, 0, False) > 0
    assert size(*long, 0, True, True) > size(*long, 0, True) > 0
    assert size(2, 2, 40, 48, 0, True) == 0 and size(0, 2, 40, 32, 0, True) == 0 and size(2, 2, 40, 32, 9, True) == 0
    for call, ptrs, n in ((forward, FWD, size(*long, 0, False)), (backward, BWD, size(*long, 0, True, True)),
                          (backward, BWD[:9] + (None,), size(*long, 0, True))):
        assert call(lib, ptrs, long) == -6
        assert call(lib, ptrs, long, workspace=0x100000, workspace_bytes=n - 1) == -6


def test_bindings_refuse():
    x, g = torch.zeros(1, 2, 8, 32), torch.zeros(2)
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_decay_fwd(x, x, x, g, None)
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_decay_bwd(x, x, x, g, None, x)
    for bad in (torch.zeros(1), torch.zeros(1, 2), torch.zeros(2, dtype=torch.float64), torch.zeros(4)[::2]):
        with pytest.raises(ValueError, match="g must be"):
            binding._check_decays("g", bad, 2, x.device)
    for scale in (0, -1.0, 1e-50):
        with pytest.raises(ValueError, match="scale"):
            binding._decay_params(x, (1, 2, 8, 32), scale, None, "bhnd", None)
    for name in ("initial_state", "final_state", "dfinal_state", "dinitial_state"):
        with pytest.raises(ValueError, match=name):
            binding._decay_params(x, (1, 2, 8, 32), None, None, "bhnd", None, **{name: torch.zeros(2, 1, 32, 32)})


@pytest.fixture
def stand_ins(monkeypatch):
    wanted = []

    def decay_bwd(prm, dims, Q, K, V, g, mask, dO, initial_state, dfinal_state, dinitial_state, dg):
        wanted.append((dg is not None, dinitial_state is not None, dO.data_ptr() % 16))
        for t in (dg, dinitial_state):
            if t is not None:
                t.fill_(1.0)
        return tuple(torch.ones_like(Q) for _ in range(3))

    monkeypatch.setattr(binding, "cotten_decay_fwd", lambda Q, *a, **kw: Q.detach() + 1.0)
    monkeypatch.setattr(binding, "_decay_backward_of", decay_bwd)
    return wanted


def test_only_wanted_gradients_and_no_second_derivatives(stand_ins):
    x = torch.randn(1, 2, 4, 16, requires_grad=True)
    g, S0 = torch.randn(2), torch.randn(1, 2, 16, 16)
    for of_g, of_S in ((False, False), (True, False), (True, True)):
        y = autograd.decay_attention(x, x, x, g.clone().requires_grad_(of_g), initial_state=S0.clone().requires_grad_(of_S))
        # an upstream gradient that begins anywhere
        (torch.cat([x.flatten()[:3], y.flatten()]) * torch.randn(3 + y.numel())).sum().backward()
        assert stand_ins.pop() == (of_g, of_S, 0)
    y = autograd.decay_attention(x, x, x, g)
    first, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad(y.sum() + first.square().sum(), x)
