"""Counts of a rotating call come from one place, which holds them to the batch: the library reads one of each sequence."""
import numpy as np
import pytest

import paper_2510_08525_amd as rl
from paper_2510_08525_amd import binding


def test_no_call_takes_counts_of_any_number():
    """Calls by address cannot know the batch of a handle, so the package has none for counts that the tensor calls check."""
    for name in ("rlkv_append_rotary", "rlkv_rotary"):
        assert not hasattr(rl, name) and not hasattr(binding, name)
        assert hasattr(rl.load_library(), name)


@pytest.mark.parametrize("counts", [[], [1], [1, 2], [1, 2, 3, 4], [[1, 2, 3]], 3, np.ones((3, 1), dtype=np.int32)])
def test_counts_of_another_number_are_refused(counts):
    cache = object.__new__(rl.Cache)
    cache.shape = dict(batch=3)
    for call in (lambda: cache.append_rotary(0, None, counts, rl.Rotary([1.0] * 8)),
                 lambda: cache.rotary(0, None, counts, rl.Rotary([1.0] * 8), None, None, None)):
        with pytest.raises(ValueError, match="batch entries"):
            call()
