"""Log-probabilities at the ends of what the calls take: numbers of rows, temperatures, distances between logits."""
from __future__ import annotations

import pytest

from paper_2509_24248_b200 import binding as sx

pytestmark = pytest.mark.gpu


def test_workspace_of_the_largest_numbers_of_rows():
    """Any number of rows is taken in parts of 1024 at most, whose workspace is the largest there is."""
    size = sx.load_library().sx_head_logprobs_ws_bytes
    most = size(1024, 300)
    for T in (1024, 2048, 2 ** 31 - 1024, 2 ** 31 - 1023, 2 ** 31 - 1):
        assert size(T, 300) == most, T
    assert 0 < size(1025, 300) < most and 0 < size(2 ** 31 - 1, 300)
