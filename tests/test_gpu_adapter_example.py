"""The brittleness example end to end: valuation, training of four subsets' adapters in the same batches, losses."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_removing_what_is_valued_costs_more_than_removing_at_random():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import subset_adapters
    losses, informative = subset_adapters.run()
    print(losses, informative, flush=True)
    # half of the data is noise: a valuation that says nothing would take half of its quarter (64 of 256 examples,
    # standard deviation 0.055) from it
    assert informative > 0.6
    assert losses["without the most valuable quarter"] > losses["without a random quarter"] > losses["all data"] - 0.1
    assert losses["all data"] < losses["no adapter"] - 0.3
