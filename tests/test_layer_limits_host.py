"""The largest sizes that the operators behind the router take, by their refusals (found before anything needs a device)."""
import os
import re

import pytest

from paper_2609_36301_b200 import binding, build

A = 4096                                                       # an address that is never read
TOO_LARGE = -8
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "more_route.h")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_most_pairs(lib):
    """A run is rounded up to whole tiles and pieces in 32-bit numbers.  Within 127 pairs of 2^31 the tiles of one expert's run came to a
    negative number, and a forward call did nothing and reported success."""
    most = int(re.search(r"#define MORE_PAIRS_MAX (0x[0-9a-f]+)", open(HEADER).read()).group(1), 16)
    assert most + 8192 <= 2 ** 31 - 1
    assert lib.more_experts_workspace(most, 8, 8, 1, 1, 0) > 0
    assert lib.more_experts_workspace(most, 8, 8, 1, 1, 1) > 0
    for T, k in ((most + 1, 1), (2 ** 31 - 1, 1), (most // 2 + 1, 2)):
        for backward in (0, 1):
            assert lib.more_experts_workspace(T, 8, 8, 2, k, backward) == TOO_LARGE
        assert lib.more_experts_path(T, 8, 8, 2, k) == TOO_LARGE
        assert lib.more_experts(A, A, A, A, A, A, T, 8, 8, 2, k, A, None, 2, A, 1 << 60, None) == TOO_LARGE
        assert lib.more_experts_backward(A, A, A, A, A, A, A, A, A, T, 8, 8, 2, k, A, A, A, A, A, 1 << 60, None) == TOO_LARGE
