"""The paged cache's calls at the ends of their ranges."""
import numpy as np
import pytest
import torch

import paged_ref as R
from gpu_util import device, note
from paper_2606_00535_amd import dreams

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = device()
    dreams.lib()
    return d


def test_fork_in_a_table_without_sequences(dev):
    """Every index is outside the table: nothing is granted."""
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
    pages = torch.zeros((3, 2, 16, 64), device=dev)
    side = torch.cuda.Stream()
    for kw in (dict(), dict(stream=side)):
        granted = torch.full((3,), 7, dtype=torch.int32, device=dev)
        torch.cuda.synchronize()
        got = dreams.pages_fork(pages, pages, z(0, 4), z(0), z(0), z(3), z(3), z(3) + 1, granted=granted, **kw)
        torch.cuda.synchronize()
        assert got is granted and got.tolist() == [0, 0, 0]
