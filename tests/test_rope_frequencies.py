"""Defaults of rope_frequencies: each scaling's own published ones."""

import pytest

import paper_2605_04084_amd as fasq


def test_yarn_takes_its_own_turns():
    """arXiv 2309.00071: pairs that turn 32 times or more are left, those that turn less than once slowed."""
    kw = dict(base=10000.0, scaling="yarn", factor=16.0, original=4096)
    assert fasq.rope_frequencies(128, **kw) == fasq.rope_frequencies(128, low=1.0, high=32.0, **kw)
    assert fasq.rope_frequencies(128, high=8.0, **kw) != fasq.rope_frequencies(128, **kw)


def test_wavelength_takes_its_own_turns():
    kw = dict(base=500000.0, scaling="wavelength", factor=8.0, original=8192)
    assert fasq.rope_frequencies(128, **kw) == fasq.rope_frequencies(128, low=1.0, high=4.0, **kw)


@pytest.mark.parametrize("scaling", ["yarn", "wavelength"])
@pytest.mark.parametrize("low,high", [(40.0, None), (2.0, 1.0), (0.0, 4.0)])
def test_turns_out_of_order(scaling, low, high):
    with pytest.raises(ValueError, match="low < high"):
        fasq.rope_frequencies(64, scaling=scaling, factor=2.0, original=2048, low=low, high=high)
