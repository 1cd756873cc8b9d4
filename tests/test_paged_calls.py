"""What the paged cache's calls check and plan on the host.  No kernel runs here."""
import types

import pytest
import torch

from paper_2606_00535_amd import dreams


def test_a_stream_of_another_device():
    """Kernels run on the current device; a stream of another one is refused."""
    stream = lambda index: types.SimpleNamespace(device=torch.device("cuda", index), cuda_stream=77)
    assert dreams._stream_on(stream(0), 0) == 77 and dreams._stream_on(stream(3), 3) == 77
    for at in (0, 2):
        with pytest.raises(ValueError, match="stream is on cuda:1"):
            dreams._stream_on(stream(1), at)
