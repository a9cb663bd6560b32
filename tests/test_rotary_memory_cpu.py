"""What a Rotary hands to the library lives as long as the Rotary: nobody else can free, move or change it."""
import ctypes

import numpy as np
import pytest

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding


def _behind(rotary):
    """The frequencies at the address that the library gets."""
    s = binding._Rotary.from_address(rotary.address)
    return list((ctypes.c_double * s.n_pairs).from_address(s.inv_freq)), s.interleaved


def test_frequencies_cannot_be_replaced():
    r = rl.Rotary([0.5] * 8, interleaved=True)
    with pytest.raises(AttributeError):
        r.inv_freq = np.ones(8)
    with pytest.raises(AttributeError):
        r.address = 0
    assert _behind(r) == ([0.5] * 8, 1)


def test_frequencies_are_the_rotarys_own():
    mine = np.arange(16, dtype=np.float64)
    r = rl.Rotary(mine)
    mine[:] = -1.0
    assert _behind(r) == (list(range(16)), 0) and list(r.inv_freq) == list(range(16))
    with pytest.raises(ValueError):
        r.inv_freq[0] = 2.0
