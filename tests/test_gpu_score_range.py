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


def ends(T, V, dtype, seed):
    """Logits of every size up to the type's largest, of both signs, both ends of it in every row; one row of -inf but for two."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.rand(T, V, generator=g) * 2 - 1) * torch.finfo(dtype).max
    x[:, 0], x[:, V - 1] = torch.finfo(dtype).max, torch.finfo(dtype).min
    x[T - 1, 2:] = float("-inf")
    x[T - 1, 1] = torch.finfo(dtype).min
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [3, 17, 40, 3000, 200001])
@pytest.mark.parametrize("temperature", [1e32, 1e37, 1e38, 3e38])
def test_distances_beyond_the_range(dtype, V, temperature):
    """Logits further apart than fp32's largest number, whose probabilities are alike at such a temperature."""
    x = ends(5, V, dtype, V).to(DEV)
    both(x, torch.tensor([[0, V - 1, V // 2]] * 5, dtype=torch.int32, device=DEV), 3, temperature)


@pytest.mark.parametrize("temperature", [2.0, 30.0])
def test_a_log_probability_within_the_range_of_a_distance_beyond_it(temperature):
    """The type's lowest value under a largest logit that counts beside it: log p is a finite number."""
    x = torch.full((2, 500), torch.finfo(torch.float32).min, device=DEV)
    x[:, 7] = 1e35
    x[1, 9] = 0.0
    both(x, torch.tensor([[3, 7, 9]] * 2, dtype=torch.int32, device=DEV), 4, temperature)


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("temperature", [1e37, 1e38])
def test_distances_beyond_the_range_through_a_head(T, temperature):
    """Logits of +-2^127 and sums of a few smaller powers of two, exact in fp32."""
    H, V = 64, 700
    g = torch.Generator().manual_seed(41)
    h, w = torch.zeros(T, H), torch.zeros(V, H)
    h[:, :2] = 2.0 ** 63
    w[:, 0] = torch.randint(-1, 2, (V,), generator=g) * 2.0 ** 64
    w[:, 1] = torch.randint(-3, 4, (V,), generator=g) * 2.0 ** 61
    w[w[:, 0] * w[:, 1] > 0, 1] = 0                              # the larger sums would leave the range
    h, w = h.to(torch.bfloat16).to(DEV), w.to(torch.bfloat16).to(DEV)
    tok = torch.randint(0, V, (T, 2), generator=g).to(torch.int32).to(DEV)
    s = sx.LogProbs(w)
    got = s.sx_head_logprobs(h, tok, top=9, temperature=temperature)
    s.check_status()
    x = h.double().cpu() @ w.double().cpu().T
    ref.check(got, ref.scores(x, tok, 9, temperature), x, temperature)
