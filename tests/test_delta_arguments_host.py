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
