"""Rotations and 8-bit rows of more than 2^32 bytes, and outputs that lie on their inputs."""
import numpy as np
import pytest
import torch

from gpu_util import device, note
from paper_2606_00535_amd import dreams
import paged_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = device()
    dreams.lib()
    return d


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_rotation_past_32_bits(dev, interleaved):
    """The last rows of a large tensor are those of a small one, in both orders of heads and rows, also in place."""
    H, N, D, far = 40, 430000, 128, 50
    freq = dreams.rope_frequencies(D, 5e5)
    x = torch.empty((1, H, N, D), dtype=torch.bfloat16, device=dev)
    assert x.numel() * 2 > 1 << 32
    x[:, :2].normal_()
    x[:, H - 2:].normal_()
    kv = R.ints([7], dev)
    note("rope_far", interleaved)
    want = dreams.rope(x[:, H - 2:, N - far:].contiguous(), freq, kv + N - far, interleaved=interleaved)
    first = dreams.rope(x[:, :2, :far].contiguous(), freq, kv, interleaved=interleaved)
    out = dreams.rope(x, freq, kv, interleaved=interleaved)
    assert torch.equal(out[:, H - 2:, N - far:], want) and torch.equal(out[:, :2, :far], first)
    rows = out.view(1, N, H, D).transpose(1, 2)       # [B,N,H,D] in memory
    rows[:, H - 2:, N - far:] = x[:, H - 2:, N - far:]
    assert dreams.rope(rows, freq, kv, interleaved=interleaved, out=rows) is rows
    assert torch.equal(rows[:, H - 2:, N - far:], want)


def test_rows_in_8_bits_past_32_bits(dev):
    """New rows and rows read back that take more than 4 GiB: their ends are those of a small call."""
    H, D, ps, N, far = 8, 128, 64, 2200 * 1024, 96
    pages = N // ps
    assert H * N * D * 2 > 1 << 32 and pages <= dreams.PAGES_MAX
    freq = dreams.rope_frequencies(D)
    new = [torch.empty((1, H, N, D), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    for t in new:
        t.fill_(1.25)
        t[:, :, N - far:].normal_()
    pool = lambda n: [torch.empty((n, H, ps, D), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2)] + [
        torch.empty((n, H, ps // 16), dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu) for _ in range(2)]
    big, small = pool(pages), pool(4)
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=dev)[None]
    zero = R.ints([0], dev)
    note("rows_far")
    dreams.paged_append_e4m3(*new, *big, table, zero, frequencies=freq)
    small_table = R.ints([[0, 1, 2, 3]], dev)
    start = (N - far) // ps * ps                      # (the small pool's rows start where a page does)
    near = [t[:, :, start:].contiguous() for t in new]
    where = torch.arange(start, N, dtype=torch.int32, device=dev)[None]
    dreams.paged_append_e4m3(*near, *small, small_table, zero, frequencies=freq, positions=where)
    n = N - start
    want = dreams.paged_read_e4m3(*small, small_table, R.ints([n], dev), n)
    got = dreams.paged_read_e4m3(*big, table, R.ints([N], dev), N)
    for a, b, t in zip(got, want, new):
        assert a.numel() * 2 > 1 << 32
        assert torch.equal(a[:, :, start:], b)
        assert torch.equal(a[0, H - 1, 5] != 0, t[0, H - 1, 5] != 0)


def test_outputs_on_their_inputs_are_refused(dev):
    freq = dreams.rope_frequencies(64)
    kv = R.ints([0, 3], dev)
    buf = torch.zeros(2 * 4 * 9 * 64 + 64, dtype=torch.bfloat16, device=dev)
    a, b = buf[:-64].view(2, 4, 9, 64), buf[64:].view(2, 4, 9, 64)
    with pytest.raises(dreams.DreamsError, match="overlap"):
        dreams.rope(a, freq, kv, out=b)
    # the two halves of one buffer's rows lie between one another's: no overlap
    both = torch.randn((2, 4, 9, 128), device=dev).bfloat16()
    want = dreams.rope(both[..., :64].contiguous(), freq, kv)
    assert torch.equal(dreams.rope(both[..., :64], freq, kv, out=both[..., 64:]), want)
    k = torch.zeros((8, 2, 16, 64), dtype=torch.bfloat16, device=dev)
    rows = torch.zeros((2, 2, 9, 64), dtype=torch.bfloat16, device=dev)
    table = R.ints(np.arange(8).reshape(2, 4), dev)
    with pytest.raises(dreams.DreamsError, match="overlap"):
        dreams.paged_append_rope(rows, rows, k, k.clone(), table, kv, freq, q=a, q_out=a)
