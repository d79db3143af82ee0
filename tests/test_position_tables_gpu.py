"""Gradients of tables of positions that are much longer than the calls that use them."""
import ctypes

import pytest
import torch

from paper_2602_06935_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,N,D,rows,offset", [(16384, 1, 256, 32768, 20000), (16384, 1, 256, 32768, 0), (16384, 1, 256, 32768, 32767),
                                               (1, 1, 3, 5000, 4999), (9, 1, 512, 70000, 1), (200, 2, 99, 4096, 4094),
                                               (300, 30, 17, 9000, 77), (7, 1, 1, 100003, 50001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_long_tables(dtype, B, N, D, rows, offset):
    """One token a call, at the front, in the middle and at the end: sums in parts and in one, zeros everywhere else.  fp32
    sums of B terms, at most B / 4 + 32 roundings in a row, and one rounding to the type."""
    gen = torch.Generator().manual_seed(B + D)
    dE = torch.randn(B, N, D, generator=gen).to(dtype)
    ids = torch.randint(0, 40, (B, N), generator=gen)
    dP = torch.full((rows, D), 7.0, dtype=dtype, device="cuda")
    dW = binding.cotten_embed_bwd(ids.cuda(), dE.cuda(), 40, dP=dP, position_offset=offset)
    alone = binding.cotten_embed_bwd(ids.cuda(), dE.cuda(), 40)
    torch.cuda.synchronize()
    assert torch.equal(dW, alone)
    got, want = dP.cpu(), dE.double().sum(0)
    half = torch.finfo(dtype).eps / 2
    slack = 2.0 ** -24 * (B / 4 + 32) * B ** 0.5 * 4 + (6e-8 if dtype is torch.float16 else 0)
    assert ((got[offset:offset + N].double() - want).abs() <= half * want.abs() * 1.01 + slack).all()
    assert (got[:offset] == 0).all() and (got[offset + N:] == 0).all()


@pytest.mark.parametrize("B", [100, 192])
def test_few_shares_are_not_cut_into_parts(B):
    """Parts (a second launch, and room for their sums) only from four on: fewer than 193 rows need no workspace."""
    gen = torch.Generator().manual_seed(B)
    dE = torch.randn(B, 4, 64, generator=gen)
    ids, g, dP = torch.zeros(B, 4, dtype=torch.int64, device="cuda"), dE.cuda(), torch.full((9, 64), 7.0, device="cuda")
    prm = binding.CottenEmbedParams(binding.COTTEN_F32, 8, 1.0, -1, 9, 3, None, 0)
    binding._check(binding.load_library().cotten_embed_bwd(ids.data_ptr(), g.data_ptr(), None, dP.data_ptr(), B, 4, 64, 40,
                                                           torch.cuda.current_stream().cuda_stream, ctypes.byref(prm)))
    torch.cuda.synchronize()
    want = dE.double().sum(0)
    assert ((dP[3:7].cpu().double() - want).abs() <= 2.0 ** -24 * (B / 4 + 32) * B ** 0.5 * 4).all()
    assert (dP[:3] == 0).all() and (dP[7:] == 0).all()


@pytest.mark.parametrize("B,N,D", [(1, 1, 64), (5, 30, 99), (90, 110, 64), (700, 3, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_positions_alone(dtype, B, N, D):
    """The gradient of the positions without the table's: the same bits, by the call and by the differentiable function."""
    from paper_2602_06935_amd.autograd import item_embedding
    gen = torch.Generator().manual_seed(B + D)
    dE = torch.randn(B, N, D, generator=gen).to(dtype).cuda()
    ids = torch.randint(0, 40, (B, N), generator=gen).cuda()
    W, P = torch.randn(40, D, generator=gen).to(dtype).cuda(), torch.randn(N + 9, D, generator=gen).to(dtype).cuda()
    both, alone = torch.full_like(P, 7.0), torch.full_like(P, 7.0)
    binding.cotten_embed_bwd(ids, dE, 40, dP=both, position_offset=2)
    assert binding.cotten_embed_bwd(ids, dE, 40, dP=alone, position_offset=2, of_table=False) is None
    got, = torch.autograd.grad(item_embedding(ids, W, P.requires_grad_(), position_offset=2), P, dE)
    assert torch.equal(both, alone) and torch.equal(both, got)
    with pytest.raises(ValueError):
        binding.cotten_embed_bwd(ids, dE, 40, of_table=False)
