"""Long keys in pages of 8 bits: up to 64 rows, spread over the workgroups in pieces of one length that a second launch merges, where
the bound of the lengths says so; on the kernel of 128 rows in pieces that merge within the launch.  Against the 64-bit
definitions of tests/paged_ref.py."""
import ctypes

import numpy as np
import pytest
import torch

import e4m3_ref as E
import paged_ref as R
from gpu_util import device, note
from paper_2606_00535_amd import dreams
from test_gpu_paged_e4m3_keys import poison
from test_gpu_paged_keys import check_rows

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


def attend(kind, rng, dev, c, q, qh, heads, dim, lens, T, window, sinks, masked, bound=0):
    """(the call, its 64-bit result): a tree, or a prompt whose second sequence has no rows."""
    B = len(lens)
    kv = R.ints(lens, dev)
    kw = dict(window=window, sinks=sinks, max_kv_len=bound or max(lens))
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


# heads, D, page, lengths, T, window, sinks, mask, bound of the lengths, spread or not: 16, 32 and 64 rows
UNLIKE = [
    ((7, 1), 128, 64, [6100, 0, 5, 2048, 700], 4, 0, 0, False, 60000, True),
    ((7, 1), 128, 16, [6100, 0, 5, 2048, 700], 4, 0, 0, False, 20000, False),
    ((4, 1), 128, 64, [8000, 10, 3333], 1, 0, 0, False, 60000, True),
    ((16, 2), 128, 16, [3900, 17, 8000], 2, 0, 0, False, 60000, True),
    ((3, 1), 64, 32, [6500, 4095, 1], 5, 0, 0, True, 60000, True),
    ((4, 1), 128, 16, [6200, 4100, 900], 14, 0, 0, True, 60000, True),
    ((4, 1), 128, 64, [6200, 4100, 900], 14, 0, 0, False, 12000, False),
    ((8, 8), 128, 64, [700, 5000, 33, 1200], 1, 0, 0, False, 60000, True),
    ((8, 4), 128, 16, [900, 3, 31, 32, 33, 500, 0, 127, 128, 129, 1, 640, 64, 15, 16, 17], 1, 0, 0, False, 20000, True),
    ((4, 4), 64, 32, [3000, 10, 500], 20, 0, 0, True, 32000, True),
    ((8, 2), 128, 64, [2000], 15, 0, 0, False, 20000, True),
    ((4, 4), 128, 64, [3000, 200], 64, 0, 0, False, 60000, False),
    ((2, 1), 64, 16, [16500], 9, 16000, 40, False, 16500, True),
]


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,ps,lens,T,window,sinks,masked,bound,spread", UNLIKE)
def test_lengths_under_their_bound(dev, heads, D, ps, lens, T, window, sinks, masked, bound, spread, kind):
    """The host knows the bound alone: pieces follow the lengths that the device finds.  Twice the same, bit for bit."""
    rng = np.random.default_rng(41)
    note("unlike", heads, D, ps, lens, T, window, sinks, masked, bound, spread, kind)
    c = E.Cache8(rng, dev, np.array(lens) + T, heads[1], ps, D, width=-(-(bound + T) // ps))
    q, qh = R.rounded(rng, (len(lens), heads[0], T, D), True, dev)
    assert spreads(q, c, kind, heads, D, T, window, sinks, bound) == spread
    run, want = attend(kind, rng, dev, c, q, qh, heads, D, lens, T, window, sinks, masked, bound)
    out, lse = run()
    R.check(out, lse, want, True, (heads, lens, kind))
    again = run()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


# heads, D, lengths, T, window, sinks, bound
FAR_NAN = [((4, 1), 128, [3000, 9], 4, 0, 0, 60000), ((4, 1), 128, [3000, 9], 8, 0, 0, 60000), ((4, 1), 128, [40, 2000], 16, 0, 0, 60000),
           ((2, 2), 64, [5000], 8, 0, 0, 60000), ((1, 1), 64, [16500], 8, 16000, 5, 16500)]


@pytest.mark.parametrize("heads,D,lens,T,window,sinks,bound", FAR_NAN)
def test_spread_nodes_out_of_sight(dev, heads, D, lens, T, window, sinks, bound):
    """Keys that are NaN and of no row, of siblings, and of slots that a window leaves to some rows."""
    rng = np.random.default_rng(42)
    B, ps = len(lens), 16
    par = R.tree(rng, B, T, 4, 3)
    dep = R.depths(par)
    for how in ("masked", "sibling", "window"):
        if how == "window" and not window:
            continue
        note("spread_nodes", heads, D, lens, T, window, how)
        c = E.Cache8(rng, dev, np.array(lens) + T, heads[1], ps, D, width=-(-(bound + T) // ps))
        q, qh = R.rounded(rng, (B, heads[0], T, D), True, dev)
        assert spreads(q, c, "verify", heads, D, T, window, sinks, bound)
        see, blind = R.ancestors(par), np.ones((B, T), bool)
        for b, L in enumerate(lens):
            if how == "window":      # seen by the nodes up to depth 1 alone
                bad = [L - window + 2]
            else:
                nodes = rng.choice(np.arange(1, T), size=max(1, T // 4), replace=False)
                if how == "masked":
                    see[b, :, nodes] = False
                bad = [L + int(n) for n in nodes]
            poison(rng, c, b, bad)
            for j in bad:
                seen = see[b, :, j - L] if j >= L else np.ones(T, bool)
                if window:
                    at = L + dep[b, j - L] if j >= L else j
                    seen = seen & ((L + dep[b] - at < window) | (at < sinks))
                blind[b] &= ~seen
        mask = torch.from_numpy(R.mask_bits(see)).to(dev) if how == "masked" else None
        out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), tree_mask=mask,
                                                 window=window, sinks=sinks, max_kv_len=bound)
        ref = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
        assert how != "masked" or blind.all()
        check_rows(out, lse, ref, True, blind, how)


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,T", [((4, 1), 128, 4), ((4, 1), 128, 8), ((4, 1), 128, 16), ((2, 2), 64, 16), ((1, 1), 64, 32)])
def test_spread_keys_that_are_nan(dev, heads, D, T, kind):
    """A score of NaN makes its row's output and log-sum-exp NaN, and no other row's; one in the prefix every row's of its
    sequence."""
    rng = np.random.default_rng(43)
    ps, lens, bound = 16, [3000, 1500], 60000
    c = E.Cache8(rng, dev, np.array(lens) + T, heads[1], ps, D, width=-(-(bound + T) // ps))
    q, qh = R.rounded(rng, (2, heads[0], T, D), True, dev)
    assert spreads(q, c, kind, heads, D, T, 0, 0, bound)
    par = R.tree(rng, 2, T, 3, 3)
    see = R.ancestors(par) if kind == "verify" else np.tril(np.ones((2, T, T), bool))
    node = T // 2

    def run():
        if kind == "verify":
            got = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), max_kv_len=bound)
            return got, R.verify(qh, c.k, c.v, c.table, lens, par, see, 0, 0, 1 / np.sqrt(D))
        got = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints(lens, dev), max_kv_len=bound)
        return got, R.prompt(qh, c.k, c.v, c.table, lens, [T, T], 0, 0, 1 / np.sqrt(D))

    lost = np.zeros((2, heads[0], T), bool)
    for b, slot in ((0, lens[0] + node), (1, 700)):
        page, r = int(c.table[b, slot // ps]), slot % ps
        c.kd.view(torch.uint8)[page, :, r, 5] = 0x7f
        c.k[page, :, r] = 0
        lost[b] |= see[b, :, node] if b == 0 else True
        (out, lse), ref = run()
        on, off = (torch.from_numpy(x).to(dev) for x in (lost, ~lost))
        assert lost.any() and not lost.all()
        assert torch.isnan(out[on]).all() and torch.isnan(lse[on]).all()
        R.check(out[off], lse[off], [x[~lost] for x in ref], True, (b, "others"))
