"""What the gated delta rule and the item embedding refuse on the host, before any device work: the pointers here are never
followed."""
import ctypes

import pytest
import torch

from paper_2602_06935_amd import binding


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def delta_params(**kw):
    p = binding.CottenDeltaParams(binding.COTTEN_F32, 0.0, -1.0, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def delta_fwd(lib, ptrs=(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, None, 0x6000), dims=(2, 2, 40, 32), **kw):
    return lib.cotten_delta_fwd(*ptrs, *dims, None, ctypes.byref(delta_params(**kw)))


def delta_bwd(lib, ptrs=(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, None, 0x6000, 0x7000, 0x8000, 0x9000, 0xa000, 0xb000),
              dims=(2, 2, 40, 32), **kw):
    return lib.cotten_delta_bwd(*ptrs, *dims, None, ctypes.byref(delta_params(**kw)))


def replaced(ptrs, i, p):
    return ptrs[:i] + (p,) + ptrs[i + 1:]


FWD = (0x1000, 0x2000, 0x3000, 0x4000, 0x5000, None, 0x6000)
BWD = FWD[:6] + (0x6000, 0x7000, 0x8000, 0x9000, 0xa000, 0xb000)
BF = binding.COTTEN_BF16


@pytest.mark.parametrize("call,ptrs", [(delta_fwd, FWD), (delta_bwd, BWD)])
def test_delta_refusals(lib, call, ptrs):
    room = dict(workspace=0x100000, workspace_bytes=1 << 40)
    for i in range(len(ptrs)):
        if i == 5:
            continue
        assert call(lib, replaced(ptrs, i, None), **room) == -1, i
        assert call(lib, replaced(ptrs, i, ptrs[i] + 2), **room) == -5, i
    fn = lib.cotten_delta_fwd if call is delta_fwd else lib.cotten_delta_bwd
    assert fn(*ptrs, 2, 2, 40, 32, None, None) == -1
    for dims in ((0, 2, 40, 32), (2, 0, 40, 32), (2, 2, 0, 32), (2, 2, -1, 32), (1 << 13, 1 << 12, 40, 32), (1, 1, 1 << 25, 16)):
        assert call(lib, ptrs, dims, **room) == -2, dims
    assert call(lib, ptrs, (1, 1, 1 << 24, 32), **room) == -2            # rows beyond 31-bit byte offsets
    assert call(lib, ptrs, (1, 64, 1 << 20, 32), layout=1, **room) == -2
    for d in (0, 8, 48, 96, 256):
        assert call(lib, ptrs, (2, 2, 40, d), **room) == -3
    assert call(lib, ptrs, dtype=3, **room) == -4
    assert call(lib, ptrs, layout=2, **room) == -2
    for bad in (float("nan"), float("inf")):
        assert call(lib, ptrs, scale=bad, **room) == -7
        assert call(lib, ptrs, eps=bad, **room) == -7
    for name in ("initial_state", "final_state", "dfinal_state", "dinitial_state", "kept"):
        assert call(lib, ptrs, **{name: 0x10004}, **room) == -5, name
    assert call(lib, ptrs, workspace=0x10004, workspace_bytes=1 << 40) == -5
    need = binding.cotten_delta_kept_bytes(2, 2, 40, 32, 0)
    assert need > 0
    assert call(lib, ptrs, kept=0x10000, kept_bytes=need - 1, **room) == -6


@pytest.mark.parametrize("call,ptrs", [(delta_fwd, FWD), (delta_bwd, BWD)])
def test_delta_refuses_what_offsets_and_grids_cannot_reach(lib, call, ptrs):
    """Rows so far apart that those of a chunk beyond a short sequence's end would wrap around; more slices than a launch has
    threads for."""
    room = dict(workspace=0x100000, workspace_bytes=1 << 60)
    for N in (1, 2, 16):
        assert call(lib, ptrs, (1, 1 << 20, N, 64), layout=1, **room) == -2, N     # 32 rows of 2^28 bytes
    for dims in ((1 << 12, 1 << 11, 1, 16), (1 << 12, (1 << 10) + 1, 20, 128)):
        assert call(lib, ptrs, dims, **room) == -2, dims


def test_embed_refuses_what_grids_cannot_reach(lib):
    def call(dims, ptrs=(0x1000, 0x2000, 0x3000, 0x4000), **kw):
        return lib.cotten_embed_bwd(*ptrs, *dims, None, ctypes.byref(embed_params(workspace_bytes=1 << 60, **kw)))
    assert call(((1 << 29) + 1, 1, 33, 100), (0x1000, 0x2000, 0x3000, None)) == -2
    assert call((2, 40, 64, 100), positions=(1 << 22) + 1) == -2


def test_delta_backward_needs_its_workspace(lib):
    alone = binding.cotten_delta_workspace_bytes(2, 2, 40, 32, 0, True)
    given = binding.cotten_delta_workspace_bytes(2, 2, 40, 32, 0, True, True)
    kept = binding.cotten_delta_kept_bytes(2, 2, 40, 32, 0)
    assert alone >= given > 0
    assert delta_bwd(lib) == -6
    assert delta_bwd(lib, workspace=0x100000, workspace_bytes=alone - 1) == -6
    assert delta_bwd(lib, workspace=0x100000, workspace_bytes=given - 1, kept=0x200000, kept_bytes=kept) == -6


def test_delta_sizes(lib):
    kept, space = binding.cotten_delta_kept_bytes, binding.cotten_delta_workspace_bytes
    assert kept(2, 2, 40, 48, 0) == 0 and kept(0, 2, 40, 32, 0) == 0 and kept(2, 2, 40, 32, 9) == 0
    assert space(2, 2, 40, 48, 0, True) == 0
    # lengths whose byte counts pass 32 bits
    assert kept(64, 8, 16384, 64, BF) > (1 << 32)
    # grows with the tokens, not with their square
    assert kept(200, 2, 64000, 64, BF) <= 1001 * kept(200, 2, 64, 64, BF)


def embed_params(**kw):
    p = binding.CottenEmbedParams(binding.COTTEN_F32, 8, 1.0, -1, 50, 0, 0x100000, 1 << 40)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("backward", [False, True])
def test_embed_refusals(lib, backward):
    fn = lib.cotten_embed_bwd if backward else lib.cotten_embed_fwd
    ptrs, dims = (0x1000, 0x2000, 0x3000, 0x4000), (2, 40, 64, 100)

    def call(ptrs=ptrs, dims=dims, **kw):
        return fn(*ptrs, *dims, None, ctypes.byref(embed_params(**kw)))

    assert fn(*ptrs, *dims, None, None) == -1
    for i in (0, 1) + (() if backward else (3,)):
        assert call(replaced(ptrs, i, None)) == -1
    if backward:
        assert call((0x1000, 0x2000, None, None)) == -1
        assert call(workspace=None) == -6
        need = binding.cotten_embed_workspace_bytes(*dims)
        assert need > 0 and call(workspace_bytes=need - 1) == -6
    assert call(replaced(ptrs, 0, 0x1004)) == -5
    for i in (1, 2, 3):
        assert call(replaced(ptrs, i, ptrs[i] + 8)) == -5
    assert call(workspace=0x100004) == -5
    assert call(dtype=3) == -4 and call(id_bytes=2) == -4
    for d in ((0, 40, 64, 100), (2, 0, 64, 100), (2, 40, 0, 100), (2, 40, 64, 0), (2, 40, 70000, 100), (2, 40, 64, 1 << 30),
              (1 << 16, 1 << 15, 64, 100)):
        assert call(dims=d, positions=1 << 20) == -2, d
    # positions that the table does not have
    assert call(positions=39) == -2 and call(position_offset=11) == -2 and call(position_offset=-1) == -2
    assert call(scale=float("nan")) == -7 and call(scale=float("inf")) == -7
    assert binding.cotten_embed_workspace_bytes(0, 1, 1, 1) == 0


def test_bindings_refuse():
    x, g = torch.zeros(1, 1, 8, 32), torch.zeros(1, 1, 8)
    with pytest.raises(ValueError):
        binding.cotten_delta_fwd(x, x, x, g, g, None)
    with pytest.raises(ValueError):
        binding.cotten_delta_bwd(x, x, x, g, g, None, x)
    with pytest.raises(ValueError):
        binding.cotten_embed_fwd(torch.zeros(1, 1, dtype=torch.int64), torch.zeros(4, 8))
    with pytest.raises(ValueError):
        binding.cotten_embed_bwd(torch.zeros(1, 1, dtype=torch.int64), torch.zeros(1, 1, 8), 4)
