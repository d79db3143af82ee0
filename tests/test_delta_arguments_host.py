"""Arguments that the bindings of the gated delta rule refuse, with tensors on the CPU behind the checks that come first."""
import pytest
import torch

from paper_2602_06935_amd import binding


def parameters(B=2, H=3, N=4, d=16, **kw):
    """The parameters that the calls build of what they are given."""
    Q, gate = torch.zeros(B, H, N, d), torch.zeros(B, H, N)
    given = dict(scale=None, eps=None, layout="bhnd", workspace=None, kept=None)
    given.update(kw)
    return binding._delta_params(Q, (B, H, N, d), (("g", gate), ("beta", gate)), **given)


def test_scales():
    """The library takes 0 and below for 1: a caller who asks for them would get another result than the formula's."""
    assert parameters().scale == 0.0 and parameters(scale=0.5).scale == 0.5
    for bad in (0, 0.0, -0.0, -1.0, -1e-30, 1e-50):
        with pytest.raises(ValueError, match="scale"):
            parameters(scale=bad)


@pytest.mark.parametrize("name", ["initial_state", "final_state", "dfinal_state", "dinitial_state"])
def test_shapes_of_states(name):
    """As many elements in another order are not taken for a state."""
    for shape in ((2, 3, 16, 16), (6, 16, 16)):
        t = torch.zeros(shape)
        assert getattr(parameters(**{name: t}), name) == t.data_ptr()
    for shape in ((3, 2, 16, 16), (2, 16, 3, 16), (1, 6, 16, 16), (6, 256), (1536,), (2, 3, 16, 8), (3, 6, 16, 16)):
        with pytest.raises(ValueError, match=name):
            parameters(**{name: torch.zeros(shape)})


def test_short_sequences_are_not_cut_into_segments():
    """Segments take a second launch and a step over each: few chunks of 32 tokens do not make up for them (a forward without
    `kept` needs a workspace for segments only)."""
    F32, BF16, F16 = binding.COTTEN_F32, binding.COTTEN_BF16, binding.COTTEN_F16
    for d in (16, 32, 64, 128):
        for dtype in (F32, BF16, F16):
            shortest = 8 if d <= 32 else 9 if d == 64 or dtype == F32 else 17
            for B, H in ((1, 1), (4, 4)):
                cut = [c for c in range(1, 40) if binding.cotten_delta_workspace_bytes(B, H, 32 * c, d, dtype, False) != 0]
                assert cut == list(range(shortest, 40)), (B, H, d, dtype)
