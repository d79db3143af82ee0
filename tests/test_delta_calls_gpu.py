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
