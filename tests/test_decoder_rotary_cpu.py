"""What of a rotation's choices is refused when it is made."""
import pytest
import torch

from paper_1905_13298_amd import decoder


def test_sections_are_whole_numbers():
    f = torch.ones(8, dtype=torch.float64)
    assert decoder.Rotary(f, sections=[torch.tensor(4), 4]).sections == (4, 4) and decoder.Rotary(f).sections is None
    for bad in ((4.0, 4.0), (4.5, 3.5), ("4", "4"), (None, 8)):
        with pytest.raises(TypeError):
            decoder.Rotary(f, sections=bad)


@pytest.mark.parametrize("window,error", [(-1, ValueError), (2 ** 31, ValueError), (16.0, TypeError), (None, TypeError)])
def test_a_window_is_refused_before_there_is_a_cache(window, error):
    with pytest.raises(error):
        decoder.DecoderLayer({}, 4, 2, 16, 128, window=window)       # (the check comes before the weights are looked at)
