"""The limits of smoke(): an error that is no number is beyond all of them, wherever it stands among the others."""
import numpy as np
import pytest

import __graft_entry__


@pytest.mark.parametrize("where", [0, 1, 2])
def test_a_nan_is_not_within_a_limit(where):
    errors = [1e-4, np.float64(2e-4), 3e-4]
    assert __graft_entry__._within(errors, 1e-3) and __graft_entry__._within({"a": 1e-3}.values(), 1e-3)
    for bad in (np.nan, np.float64(np.nan), np.inf, 2e-3):
        errors[where] = bad
        assert not __graft_entry__._within(errors, 1e-3)


def test_smoke_compares_with_nothing_else():
    with open(__graft_entry__.__file__) as f:
        assert "assert max(" not in f.read()
