"""Gradients of tables that no launch reaches are refused before anything is enqueued (the pointers are never followed)."""
import ctypes

import pytest

from paper_2602_06935_amd import binding


@pytest.mark.parametrize("dims,positions", [((2, 40, 65536, (1 << 30) - 1), 50), ((200, 50, 65536, (1 << 30) - 1), 50),
                                            ((2, 40, 20000, (1 << 24)), 50), ((2, 40, 65536, 100), 1 << 22)])
def test_refusals(dims, positions):
    lib = binding.load_library()
    prm = binding.CottenEmbedParams(binding.COTTEN_F32, 8, 1.0, -1, positions, 0, 0x100000, 1 << 60)
    assert lib.cotten_embed_bwd(0x1000, 0x2000, 0x3000, 0x4000, *dims, None, ctypes.byref(prm)) == -2
