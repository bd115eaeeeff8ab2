"""Rotary's parameters without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_1912_12607_amd import positions  # noqa: E402


@pytest.mark.parametrize("name,value", [("rot", 4), ("layout", "interleaved"), ("amplitude", 2.0), ("frequencies", torch.ones(4, dtype=torch.float64))])
def test_parameters_are_not_replaced(name, value):
    """Calls keep descriptors and frequencies: an assignment would reach some of them only."""
    r = positions.Rotary(8)
    with pytest.raises(AttributeError):
        setattr(r, name, value)


def test_frequencies_are_the_callers_copy():
    own = torch.ones(4, dtype=torch.float64)
    r = positions.Rotary(8, frequencies=own)
    own.zero_(), r.frequencies.zero_()
    assert r.frequencies.tolist() == [1.0] * 4 and r.rot == 8 and r.layout == "half" and r.amplitude == 1.0
