"""Arguments that the bindings of the embedding refuse before the library sees them."""
import pytest
import torch

from paper_2602_06935_amd import binding


def test_numbers_beyond_32_bits():
    """ctypes hands on the lower 32 bits of a number: 2^32 would be the padding id 0, or the first position."""
    ids, W = torch.zeros(2, 3, dtype=torch.int64), torch.zeros(5, 8)

    def params(padding_idx=None, positions=0, position_offset=0):
        return binding._embed_params(ids, W, 1.0, padding_idx, positions, position_offset)

    assert params().padding_idx == -1
    p = params(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)
    assert (p.padding_idx, p.positions, p.position_offset) == (2 ** 31 - 1,) * 3
    for bad in (dict(padding_idx=2 ** 32), dict(padding_idx=2 ** 31), dict(padding_idx=-1), dict(positions=2 ** 32 + 50),
                dict(position_offset=2 ** 32 + 3), dict(position_offset=3 - 2 ** 32)):
        with pytest.raises(ValueError):
            params(**bad)


def test_tables_beyond_32_bits(monkeypatch):
    """A table of 2^32 + 5 rows is not one of 5 (tensors without memory stand in)."""
    monkeypatch.setattr(binding, "_check_table", lambda *a: None)
    ids = torch.zeros(2, 3, dtype=torch.int64, device="meta")
    with pytest.raises(ValueError, match="rows"):
        binding.cotten_embed_fwd(ids, torch.empty(2 ** 32 + 5, 1, device="meta"))
    with pytest.raises(ValueError, match="rows"):
        binding.cotten_embed_bwd(ids, torch.empty(2, 3, 1, device="meta"), 2 ** 32 + 5)
