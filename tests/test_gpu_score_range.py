"""Log-probabilities at the ends of what the calls take: numbers of rows, temperatures, distances between logits."""
from __future__ import annotations

import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import score_ref as ref
from tests.test_gpu_logprobs import TYPES, given, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def both(x, tok, top, temperature):
    s = sx.LogProbs()
    got = s.sx_logprobs(x, tok, top=top, temperature=temperature)
    s.check_status()
    ref.check(got, ref.scores(x, tok, top, temperature), x, temperature)


def test_workspace_of_the_largest_numbers_of_rows():
    """Any number of rows is taken in parts of 1024 at most, whose workspace is the largest there is."""
    size = sx.load_library().sx_head_logprobs_ws_bytes
    most = size(1024, 300)
    for T in (1024, 2048, 2 ** 31 - 1024, 2 ** 31 - 1023, 2 ** 31 - 1):
        assert size(T, 300) == most, T
    assert 0 < size(1025, 300) < most and 0 < size(2 ** 31 - 1, 300)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("temperature", [1e30, 1e38, 3e38])
def test_infinite_logits_at_the_largest_temperatures(dtype, temperature):
    """+inf anywhere in a row, behind a lane's first group of it too, leaves no probabilities; masks of -inf do."""
    x = make(8, 9000, dtype, 31).clone()
    for r, at in enumerate((0, 700, 3000, 5555, 8999)):
        x[r, at] = float("inf")
    x[5, ::2] = float("-inf")
    x[6] = float("-inf")
    both(x, given(8, 9000, 3, 32), 6, temperature)
