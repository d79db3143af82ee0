"""What the step of a beam search refuses on the host, before any device work: the pointers here are never followed."""
import ctypes

import pytest
import torch

from paper_2602_06935_amd import binding


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


PTRS = (0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x6000)


def select(lib, ptrs=PTRS, dims=(2, 4, 100), **kw):
    p = binding.CottenBeamParams(0, 0, 0x10000, 1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return lib.cotten_beam_select(*ptrs, *dims, None, ctypes.byref(p))


def test_select_refusals(lib):
    assert lib.cotten_beam_select(*PTRS, 2, 4, 100, None, None) == -1
    for i in range(6):
        if i != 2:
            assert select(lib, PTRS[:i] + (None,) + PTRS[i + 1:]) == -1, i
            assert select(lib, PTRS[:i] + (PTRS[i] + 2,) + PTRS[i + 1:]) == -5, i
    for dims in ((0, 4, 100), (2, 0, 100), (2, 4, 0), (2, 33, 100), (1 << 20, 4, 100), (2, 4, 1 << 30)):
        assert select(lib, dims=dims) == -2, dims
    assert select(lib, dtype=3) == -4
    assert select(lib, pad=100) == -7 and select(lib, pad=-1) == -7
    assert select(lib, workspace=0x10008) == -5 and select(lib, workspace=None) == -6
    need = binding.cotten_beam_workspace_bytes(2, 4, 100)
    assert need > 0 and select(lib, workspace_bytes=need - 1) == -6
    assert binding.cotten_beam_workspace_bytes(2, 33, 100) == 0


def test_reorder_refusals(lib):
    assert lib.cotten_beam_reorder(None, 0x1000, 2, 4, 64, None) == -1
    assert lib.cotten_beam_reorder(0x1000, None, 2, 4, 64, None) == -1
    assert lib.cotten_beam_reorder(0x1000, 0x2002, 2, 4, 64, None) == -5
    for B, K, n in ((0, 4, 64), (2, 0, 64), (2, 33, 64), (2, 4, 0), (2, 4, 1 << 40), (1 << 20, 4, 64)):
        assert lib.cotten_beam_reorder(0x1000, 0x2000, B, K, n, None) == -2, (B, K, n)


def test_bindings_refuse():
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_beam_select(torch.zeros(2, 4, 10), torch.zeros(2, 4))
    with pytest.raises(ValueError, match="GPU"):
        binding.cotten_beam_reorder(torch.zeros(2, 4, 10), torch.zeros(2, 4, dtype=torch.int32))
    dev = torch.device("cpu")
    for t in (torch.zeros(4, 2), torch.zeros(2, 4, dtype=torch.float64), torch.zeros(4, 2).t()):
        with pytest.raises(ValueError, match="scores"):
            binding._of_beams("scores", t, torch.float32, (2, 4), dev)
