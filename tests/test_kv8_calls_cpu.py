"""What the Python side of the 8-bit cache refuses before it looks for a device."""
from __future__ import annotations

import pytest
import torch

from paper_2509_24248_b200 import binding as sx
from tests import kv8_ref as ref


@pytest.mark.parametrize("name", ["group_start", "prefix_len"])
def test_half_a_group_is_refused(name):
    """group_start and prefix_len belong together: neither is silently ignored."""
    kv = ref.make_cache(2, 2, 64, 16, [20, 20], 0, groups=[0, 2], prefix=[10])
    del kv[name]
    with pytest.raises(sx.SxError, match="group_start and prefix_len"):
        sx.KV8(kv)
