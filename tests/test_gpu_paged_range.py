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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,heads,D,lens,N", [("prompt", (24, 8), 64, [0, 0, 0], 187), ("prompt", (32, 8), 128, [0], 300),
                                                 ("prompt", (4, 1), 128, [700, 20], 100), ("verify", (8, 2), 128, [1500, 3], 16),
                                                 ("verify", (4, 4), 64, [900], 60), ("verify", (8, 1), 128, [500, 0], 60)])
def test_bounds_of_the_prefix(dev, kind, heads, D, lens, N, dtype):
    """max_kv_len plans the work and nothing else: unknown in a wide table, exact, that of no prefix (too small where there is
    one), too large.  Without a prefix, its bound leaves the rows in one piece, which a wide table's does not."""
    rng = np.random.default_rng(51)
    bf16, B, ps = dtype == "bf16", len(lens), 16
    width = 32768 // ps
    note("bounds", kind, dtype, heads, D, lens, N)
    c = R.Cache(rng, dev, np.array(lens) + N, heads[1], ps, D, bf16, width=width)
    q, qh = R.rounded(rng, (B, heads[0], N, D), bf16, dev)
    par = R.tree(rng, B, N) if kind == "verify" else None
    if kind == "verify":
        ref = R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D))
        call = lambda **kw: dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), R.ints(par, dev), **kw)
        size = dreams.paged_verify_attn_workspace_size
    else:
        ref = R.prompt(qh, c.k, c.v, c.table, lens, [N] * B, 0, 0, 1 / np.sqrt(D))
        call = lambda **kw: dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), **kw)
        size = dreams.paged_prompt_attn_workspace_size
    for bound in (0, max(1, max(lens)), 1, 3, 5000, width * ps - N):
        R.check(*call(max_kv_len=bound), ref, bf16, bound)
    if bf16 and max(lens) == 0:
        assert size(dreams.paged_desc(q, c.kd, c.vd, c.tabled)) > 0
        assert size(dreams.paged_desc(q, c.kd, c.vd, c.tabled, max_kv_len=1)) == 0
