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


def test_a_bound_of_no_prefix_is_always_accepted():
    """max_kv_len = 1, also where the rows fill the table (0 means unknown)."""
    import ctypes
    n = ctypes.c_size_t(0)
    lib = dreams.lib()
    desc = lambda rows, bound: dreams.PagedDesc(2, 8, 2, 128, rows, 100, 16, 4, bound, 1, 0, 0, dreams.DREAMS_BF16, 0.1, 0)
    for size in (lib.dreams_paged_verify_attn_workspace_size, lib.dreams_paged_prompt_attn_workspace_size):
        for rows in (1, 60, 62, 63, 64):
            for bound, status in ((0, 0), (1, 0), (64 - rows, 0), (max(64 - rows, 1) + 1, -1), (-1, -1)):
                assert size(ctypes.byref(desc(rows, bound)), ctypes.byref(n)) == status, (rows, bound)
