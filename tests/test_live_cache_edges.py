"""CPU checks of the live-cache calls: what their kernels may use, and workspace sizes at the ends of the range."""
import os

import pytest

from test_live_cache import pk  # noqa: F401  (fixture)

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_26219_b200", "csrc")


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.startswith(("attention", "cache", "live"))))
def test_no_read_only_loads(name):
    """The kernels come onto the SMs while the one in front of them still writes what they will read (dependent launches), so
    loads that ask for memory that does not change while the kernel is there are not theirs to make."""
    text = open(os.path.join(CSRC, name)).read()
    assert "__ldg" not in text and "global.nc" not in text and "__restrict__" not in text
