"""Calls of the gated delta rule beside the ordinary ones of test_delta_gpu.py, against the same definition in 64 bits."""
import pytest
import torch

from delta_reference import DTYPES, check, inputs, reference
from test_delta_gpu import NAMES, back, backward, both, forward, lay

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_upstream_gradients_that_begin_anywhere(dtype):
    """Outputs and states in a concatenation behind three other values: their gradients are views off 16-byte boundaries."""
    from paper_2602_06935_amd.autograd import gated_delta_attention
    x = inputs(2, 2, 45, 32, DTYPES[dtype], seed=40, states=True)
    ref = reference(x)
    leaves = [x[n].cuda().requires_grad_() for n in ("q", "k", "v", "g", "beta", "S0")]
    O, S1 = gated_delta_attention(*leaves[:5], initial_state=leaves[5], return_state=True)
    front = leaves[0].flatten()[:3]
    loss = (torch.cat([front * 0, O.flatten()])[3:] * x["dO"].cuda().flatten()).sum()
    loss = loss.float() + (torch.cat([front.float() * 0, S1.flatten()])[3:] * x["dS1"].cuda().flatten()).sum()
    for n, t in zip(NAMES + ("dS0",), torch.autograd.grad(loss, leaves)):
        check(n, t, ref[n])


def in_32_bits(x):
    """The definition token by token in 32 bits on the CPU, gradients by differentiating it."""
    q, k, v, g, beta = leaves = [x[n].detach().clone().requires_grad_() for n in ("q", "k", "v", "g", "beta")]
    qn, kn = (t / (t.square().sum(-1, keepdim=True) + 1e-6).sqrt() for t in (q, k))
    S, o = torch.zeros(*q.shape[:2], q.shape[3], q.shape[3]), []
    for t in range(q.shape[2]):
        S = g[:, :, t, None, None].exp() * S
        e = v[:, :, t] - (kn[:, :, t, :, None] * S).sum(-2)
        S = S + kn[:, :, t, :, None] * (beta[:, :, t, None] * e).unsqueeze(-2)
        o.append((qn[:, :, t, :, None] * S).sum(-2))
    O = torch.stack(o, 2)
    return dict(zip(NAMES, torch.autograd.grad(O, leaves, x["dO"])), O=O.detach(), S1=S.detach())


@pytest.mark.parametrize("d", [32, 64])
def test_fp32_is_as_near_as_the_definition_in_32_bits(d):
    """Pieces of operands leave out less than half a rounding of a product, and of either sign, so results are about as far from
    64 bits as a computation that rounds every product and sum to 32: on the average of the outputs, a tenth further at most."""
    x = inputs(16, 2, 200, d, torch.float32, seed=41)
    ref, plain = reference(x), in_32_bits(x)
    O, S1, held = forward(x, kept=True)
    got = dict(backward(x, kept=held), O=O, S1=S1)
    names = NAMES + ("O", "S1")

    def off(t):
        return sum(((t[n].cpu().double() - ref[n]).norm() / ref[n].norm()).item() for n in names) / len(names)

    assert off(got) <= 1.1 * off(plain), (off(got), off(plain))


@pytest.mark.parametrize("N", [1, 2, 5, 6])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_recurrence(dtype, d, layout, N):
    """Calls of few tokens and few slices, which run token by token: strides of both layouts, masks, states."""
    x = inputs(3, 2, N, d, DTYPES[dtype], seed=50 + d + N, mask="holes" if N > 1 else None, states=True)
    ref = reference(x, scale=0.5, grads=False)
    O, S1, _ = forward(x, layout, scale=0.5)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("d,slices,N", [(64, 2051, 1), (64, 2051, 7), (128, 1031, 3), (128, 1031, 10), (32, 4099, 2), (16, 4097, 10)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_recurrence_of_many_slices(dtype, d, slices, N, layout):
    """More than 4096 waves, four to a workgroup, the last of which is not full but for d = 128; up to ten tokens."""
    B = {2051: 293, 4097: 241}.get(slices, slices)
    x = inputs(B, slices // B, N, d, DTYPES[dtype], seed=60 + d + N, mask="holes" if N > 1 else None, states=True)
    ref = reference(x, scale=0.5, grads=False)
    O, S1, _ = forward(x, layout, scale=0.5)
    check("O", O, ref["O"])
    check("S1", S1, ref["S1"])
