"""Frequencies of rotary positions that cannot be had are refused (no GPU needed)."""
import pytest

from test_tree_abi import cdsl  # noqa: F401

torch = pytest.importorskip("torch")


def test_frequencies_that_are_not_finite_are_refused(cdsl):
    """A factor so small that a frequency over it passes 64 bits' range."""
    t = torch.full((32,), 77, dtype=torch.int64)
    for factor in (5e-324, 1e-309):
        assert cdsl.lib().cdsl_rope_turns(64, 1e4, factor, 4096, 1.0, 1e9, t.data_ptr()) == cdsl.CDSL_EINVAL
        assert "cdsl_rope_turns" in cdsl.cdsl_last_error(None)
    with pytest.raises(cdsl.CdslError):
        cdsl.Rope(64, factor=5e-324, original_len=4096, high=1e9, device="cpu")
    assert cdsl.lib().cdsl_rope_turns(64, 1e4, 0.25, 4096, 1.0, 1e9, t.data_ptr()) == 0
