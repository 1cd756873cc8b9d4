"""Long keys in pages of 8 bits, on the kernel of 128 rows: in pieces that merge within the launch, against the 64-bit definitions
of tests/paged_ref.py."""
import ctypes

import numpy as np
import pytest
import torch

import e4m3_ref as E
import paged_ref as R
from gpu_util import device, note
from paper_2606_00535_amd import dreams

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = device()
    dreams.lib()
    return d


def workspace_bytes(q, c, kind, window, sinks, max_kv_len, splits):
    desc, _ = dreams._paged_desc8(q, *c.pages, window, sinks, max_kv_len, splits, None)
    n, lib = ctypes.c_size_t(0), dreams.lib()
    size = lib.dreams_paged_prompt_attn_e4m3_workspace_size if kind == "prompt" else lib.dreams_paged_verify_attn_e4m3_workspace_size
    assert size(ctypes.byref(desc), ctypes.byref(n)) == 0
    return n.value


def rows_of(dim, heads, T):
    """Rows of a workgroup."""
    rows = heads[0] // heads[1] * T
    return 16 if rows <= 16 else 32 if rows <= 32 else 64 if rows <= 64 and dim == 128 else 128


def spreads(q, c, kind, heads, dim, T, window, sinks, max_kv_len):
    """Whether the library spreads the call's keys in pieces of one length: the workspace is of their rows alone."""
    rows, units = rows_of(dim, heads, T), q.shape[0] * heads[1]
    if rows == 128:
        return False
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    wgs = max(2 * cus if rows == 64 else cus, 2 * units)
    return (workspace_bytes(q, c, kind, window, sinks, max_kv_len, 0) ==
            dreams.WORKSPACE_COUNTER_BYTES + wgs * rows * (dim * 4 + 8))


def attend(kind, rng, dev, c, q, qh, heads, dim, lens, T, window, sinks, masked, splits=0):
    """(the call, its 64-bit result): a tree, or a prompt whose second sequence has no rows."""
    B = len(lens)
    kv = R.ints(lens, dev)
    kw = dict(window=window, sinks=sinks, max_kv_len=max(lens), num_splits=splits)
    if kind == "prompt":
        rows = [T if b != 1 else 0 for b in range(B)]
        rl = R.ints(rows, dev)
        return (lambda **more: dreams.paged_prompt_attn_e4m3(q, *c.pages, kv, rl, **{**kw, **more}),
                R.prompt(qh, c.k, c.v, c.table, lens, rows, window, sinks, 1 / np.sqrt(dim)))
    par = R.tree(rng, B, T)
    see = R.ancestors(par)
    if masked:
        see &= rng.random(see.shape) < 0.5
    mask, pard = torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None, R.ints(par, dev)
    return (lambda **more: dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=pard, tree_mask=mask, **{**kw, **more}),
            R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(dim)))


# heads, D, page, lengths, T, window, sinks, mask: 65 to 128 rows of 128 columns, 33 to 128 of 64
MANY_ROWS = [
    ((7, 1), 128, 64, [20000, 300, 9000], 15, 0, 0, False),
    ((8, 1), 128, 16, [16400], 16, 0, 0, True),
    ((10, 2), 128, 32, [17000, 12], 13, 12000, 40, False),
    ((1, 1), 128, 64, [18000, 18000, 0, 31], 128, 0, 0, False),
    ((2, 2), 64, 64, [20000, 17], 33, 0, 0, False),
    ((5, 1), 64, 16, [9000, 8500, 1], 20, 0, 0, True),
    ((40, 1), 64, 64, [18000], 3, 17000, 5, False),
    ((3, 3), 64, 32, [6789, 6000], 38, 0, 0, False),
]


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,ps,lens,T,window,sinks,masked", MANY_ROWS)
def test_many_rows_behind_long_keys(dev, heads, D, ps, lens, T, window, sinks, masked, kind):
    """Pieces as over bf16 pages, whose merge gives the same bits every time; and the same rows in one piece."""
    rng = np.random.default_rng(40)
    note("many_rows", heads, D, ps, lens, T, window, sinks, masked, kind)
    c = E.Cache8(rng, dev, np.array(lens) + T, heads[1], ps, D)
    q, qh = R.rounded(rng, (len(lens), heads[0], T, D), True, dev)
    assert rows_of(D, heads, T) == 128
    run, want = attend(kind, rng, dev, c, q, qh, heads, D, lens, T, window, sinks, masked)
    # (one piece takes no workspace; two and more take their rows)
    assert workspace_bytes(q, c, kind, window, sinks, max(lens), 1) == 0
    two, chosen = (workspace_bytes(q, c, kind, window, sinks, max(lens), n) for n in (2, 0))
    assert chosen >= 4 * (two - dreams.WORKSPACE_COUNTER_BYTES)
    out, lse = run()
    R.check(out, lse, want, True, (heads, lens, kind))
    again = run()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    R.check(*run(num_splits=1), want, True, (heads, lens, kind, "whole"))
