"""Pages of 8 bits: keys that are NaN, pools past 32 bits, workspaces, and the memory of calls on a stream of their own."""
import numpy as np
import pytest
import torch

import e4m3_ref as E
import paged_ref as R
from gpu_util import device, note
from paper_2606_00535_amd import dreams
from test_gpu_paged_keys import PROMPTS, TREES, check_rows
from test_gpu_paged_streams import stream_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    d = device()
    dreams.lib()
    return d


def poison(rng, c, b, slots):
    """Codes of a sequence's keys become NaN or the largest ones, element by element (their block's scale stays); the
    definition's copy has zeros there."""
    ps = c.k.shape[2]
    for j in slots:
        page, r = int(c.table[b, j // ps]), j % ps
        bad = rng.choice(np.array([0x7f, 0xff, 0x7e, 0xfe], np.uint8), size=c.k[page, :, r].shape)
        bad[:, 0] = 0x7f
        c.kd.view(torch.uint8)[page, :, r] = torch.from_numpy(bad).to(c.kd.device)
        c.k[page, :, r] = 0


# few heads behind long prefixes, whose keys are spread in pieces of one length
SPREAD = [((4, 1), 128, [3000, 9], 4, 0, 0, 0), ((2, 2), 64, [5000], 8, 700, 5, 0)]


@pytest.mark.parametrize("heads,D,lens,T,window,sinks,splits", TREES + SPREAD)
def test_nodes_out_of_sight(dev, heads, D, lens, T, window, sinks, splits):
    """Keys of nodes that a mask hides from every row, of siblings, and of slots that a window leaves to some rows."""
    rng = np.random.default_rng(34)
    B, ps = len(lens), 16
    note("nodes_e4m3", heads, D, lens, T, window, sinks, splits)
    par = R.tree(rng, B, T, 4, 3)
    dep = R.depths(par)
    for how in ("masked", "sibling", "window"):
        if how == "window" and not window:
            continue
        c = E.Cache8(rng, dev, np.array(lens) + T, heads[1], ps, D)
        q, qh = R.rounded(rng, (B, heads[0], T, D), True, dev)
        see = R.ancestors(par)
        blind = np.ones((B, T), bool)
        for b, L in enumerate(lens):
            if how == "window":      # seen by the nodes up to depth 1 alone
                bad = [j for j in (L - window + 2,) if sinks <= j < L]
            else:
                nodes = rng.choice(np.arange(1, T), size=max(1, T // 6), replace=False)
                if how == "masked":
                    see[b, :, nodes] = False
                bad = [L + int(n) for n in nodes]
            poison(rng, c, b, bad)
            for j in bad:
                seen = see[b, :, j - L] if j >= L else np.ones(T, bool)
                at = L + dep[b, j - L] if j >= L else j
                if window:
                    seen = seen & ((L + dep[b] - at < window) | (at < sinks))
                blind[b] &= ~seen
        mask = torch.from_numpy(R.mask_bits(see)).to(dev) if how == "masked" else None
        out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), tree_mask=mask,
                                                 window=window, sinks=sinks, num_splits=splits)
        torch.cuda.synchronize()
        ref = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
        assert how != "masked" or blind.all()
        check_rows(out, lse, ref, True, blind, how)


@pytest.mark.parametrize("heads,D,lens,N,window,sinks,splits", PROMPTS)
def test_later_rows_and_keys_behind_a_window(dev, heads, D, lens, N, window, sinks, splits):
    rng = np.random.default_rng(35)
    B, ps = len(lens), 16
    note("prompt_e4m3", heads, D, lens, N, window, sinks, splits)
    c = E.Cache8(rng, dev, np.array(lens) + N, heads[1], ps, D)
    q, qh = R.rounded(rng, (B, heads[0], N, D), True, dev)
    blind = np.ones((B, N), bool)
    for b, L in enumerate(lens):
        bad = [L + N - 1, L + N - 2, L + 3 * N // 4]
        if window and L > window:
            bad.append(L - window + 2)           # the first row's alone, and the second's
        poison(rng, c, b, bad)
        for j in bad:
            at = L + np.arange(N)
            blind[b] &= ~((at >= j) & ((at - j < window) if window else True))
    out, lse = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints(lens, dev), window=window, sinks=sinks, num_splits=splits)
    torch.cuda.synchronize()
    ref = R.prompt(qh, c.k, c.v, c.table, lens, [N] * B, window, sinks, 1 / np.sqrt(D))
    check_rows(out, lse, ref, True, blind, "prompt")


@pytest.mark.parametrize("kind,heads,D,L,T,splits", [
    ("verify", (4, 4), 128, 90, 16, 0), ("verify", (4, 1), 64, 900, 8, 4), ("verify", (4, 1), 128, 3000, 4, 0),
    ("verify", (2, 2), 128, 900, 60, 4), ("verify", (4, 2), 64, 300, 60, 0), ("prompt", (4, 4), 128, 0, 20, 0),
    ("prompt", (4, 2), 64, 30, 150, 0), ("prompt", (2, 1), 128, 1500, 150, 4)])
def test_seen_keys_that_are_nan(dev, kind, heads, D, L, T, splits):
    """A score of NaN makes its row's output and log-sum-exp NaN, and no other row's."""
    rng = np.random.default_rng(36)
    ps = 16
    c = E.Cache8(rng, dev, [L + T], heads[1], ps, D)
    q, qh = R.rounded(rng, (1, heads[0], T, D), True, dev)
    par = R.tree(rng, 1, T, 4, 3)
    node = T // 2 if kind == "verify" else T - 9
    see = R.ancestors(par) if kind == "verify" else np.tril(np.ones((T, T), bool))[None]
    page, r = int(c.table[0, (L + node) // ps]), (L + node) % ps
    c.kd.view(torch.uint8)[page, :, r, 5] = 0x7f
    c.k[page, :, r] = 0
    lost = np.broadcast_to(see[0, :, node], (heads[0], T))[None]
    if kind == "verify":
        out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints([L], dev), parent=R.ints(par, dev), num_splits=splits)
        ref = R.verify(qh, c.k, c.v, c.table, [L], par, see, 0, 0, 1 / np.sqrt(D))
    else:
        out, lse = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints([L], dev), num_splits=splits)
        ref = R.prompt(qh, c.k, c.v, c.table, [L], [T], 0, 0, 1 / np.sqrt(D))
    torch.cuda.synchronize()
    on, off = (torch.from_numpy(np.ascontiguousarray(x)).to(dev) for x in (lost, ~lost))
    assert lost.any() and not lost.all()
    assert torch.isnan(out[on]).all() and torch.isnan(lse[on]).all()
    R.check(out[off], lse[off], [x[~lost] for x in ref], True, "others")


def test_a_pool_past_32_bits(dev):
    """Codes more than 2^32 bytes into a pool (and, as a view, scales too): append, commit, read, fork, attention."""
    D, ps, H, T = 128, 16, 8, 5
    rng = np.random.default_rng(37)
    page = H * ps * D
    P = (1 << 32) * 5 // 4 // page
    k, v = (torch.empty((P, H, ps, D), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2))
    near = 64                                               # pages whose scales are 80 MiB apart
    few = (1 << 32) * 5 // 4 // near // 16 * 16
    for far_scales in (False, True):
        if far_scales:      # a smaller pool whose scales lie far apart
            pages = [torch.empty((near, H, ps, D), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2)]
            scales = [torch.empty(near * few, dtype=torch.uint8, device=dev).as_strided((near, H, 1), (few, 1, 1))
                      .view(torch.float8_e8m0fnu) for _ in range(2)]
            n = near
        else:
            pages, n = [k, v], P
            scales = [torch.empty((P, H, 1), dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu) for _ in range(2)]
        table = np.array([[n - 1, 3, n - 9, n // 2, n - 2, 1, n - 37, 0]], np.int32)
        tab, zero = R.ints(table, dev), R.ints([0], dev)
        small = E.Pool8(rng, dev, 1, 8, H, ps, D)           # the same rows in a pool of 8 pages, by the definition
        order = np.arange(8, dtype=np.int32)
        new, newh = E.spread_rows(rng, (2, 1, H, 100, D), dev, True)
        dreams.paged_append_e4m3(new[0], new[1], *pages, *scales, tab, zero)
        for half in range(2):
            for g in range(H):
                small.append(half, 0, g, order, 0, newh[half, 0, g])
        slots = [small.slots(half, 0, order, 8 * ps) for half in range(2)]
        host = [x.reshape(H, 8, ps, D).transpose(1, 0, 2, 3).copy() for x in slots]
        for x in host:
            x.reshape(8, H, ps, D)[6, :, 4:] = 0            # (slots past the rows)
        got = dreams.paged_read_e4m3(*pages, *scales, tab, R.ints([100], dev), 100)
        for x, y in zip(got, slots):
            assert np.array_equal(x[0].double().cpu().numpy(), y[:, :100])
        lens, rows = [70], 21
        q, qh = R.rounded(rng, (1, 2 * H, T, D), True, dev)
        par = R.tree(rng, 1, T)
        out, lse = dreams.paged_verify_attn_e4m3(q, *pages, *scales, tab, R.ints(lens, dev), parent=R.ints(par, dev))
        R.check(out, lse, R.verify(qh, *host, order[None], lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D)), True, "far")
        q, qh = R.rounded(rng, (1, 2 * H, 100, D), True, dev)    # 200 rows a KV head: the kernel of many rows
        out, lse = dreams.paged_prompt_attn_e4m3(q, *pages, *scales, tab, zero)
        R.check(out, lse, R.prompt(qh, *host, order[None], [0], [100], 0, 0, 1 / np.sqrt(D)), True, "far prompt")
        # a move between far pages
        for half in range(2):
            for g in range(H):
                small.commit(half, 0, g, order, 60, [0, 30], 1)
        kept = dreams.paged_kv_commit_e4m3(*pages, *scales, tab, R.ints([60], dev), R.ints([[0, 30]], dev), R.ints([1], dev))
        assert kept.tolist() == [62]
        got = dreams.paged_read_e4m3(*pages, *scales, tab, kept, 62)
        for half in range(2):
            assert np.array_equal(got[half][0].double().cpu().numpy(), small.slots(half, 0, order, 62))
        assert n <= dreams.PAGES_MAX                        # a fork of a far, partly filled page
        ref = torch.ones(n, dtype=torch.int32, device=dev)
        ref[n - 5] = 0
        tab2 = torch.cat((tab[:, :5], torch.full_like(tab[:, :5], -1)))
        count, kv = R.ints([5, 0], dev), R.ints([70, 0], dev)
        granted = dreams.pages_fork_e4m3(*pages, *scales, tab2, count, kv, ref, R.ints([0], dev), R.ints([1], dev))
        assert granted.tolist() == [1] and tab2[1].tolist() == table[0, :4].tolist() + [n - 5]
        got = dreams.paged_read_e4m3(*pages, *scales, tab2, kv, 70)
        for x in got:
            assert torch.equal(x[0], x[1])


def test_workspaces(dev):
    """A caller's workspace: too small is refused, its counters are left zero; two graphs and eager calls take turns with it.
    In pieces that merge within the call, and with a second launch that merges."""
    rng = np.random.default_rng(38)
    D, lens = 128, [2000, 1900]
    for (Hq, Hkv), T, splits in (((4, 2), 60, 8), ((4, 2), 1, 0), ((16, 2), 60, 8)):
        c = E.Cache8(rng, dev, np.array(lens) + T, Hkv, 32, D)
        q, qh = R.rounded(rng, (2, Hq, T, D), True, dev)
        par, kv = R.tree(rng, 2, T), R.ints(lens, dev)
        pard = R.ints(par, dev)
        desc, _ = dreams._paged_desc8(q, *c.pages, 0, 0, 0, splits, None)
        n = dreams.ctypes.c_size_t()
        assert dreams.lib().dreams_paged_verify_attn_e4m3_workspace_size(dreams.ctypes.byref(desc), dreams.ctypes.byref(n)) == 0
        n = n.value
        assert n > 65536
        ws = torch.zeros(n, dtype=torch.uint8, device=dev)
        call = lambda room, **kw: dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=pard, num_splits=splits, workspace=room,
                                                                **kw)
        want = R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D))
        for _ in range(2):
            R.check(*call(ws), want, True, "workspace")
            dreams.workspace_status(ws)
            assert not ws[:65536].any()
        for small in (ws[:n - 256], ws[:0]):
            with pytest.raises(dreams.DreamsError) as e:
                call(small)
            assert e.value.status == dreams.DREAMS_ERR_WORKSPACE
        graphs, outs = [], []
        for scale in (None, 0.3):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                outs.append(call(ws, scale=scale))
        eager = [[x.clone() for x in call(ws, scale=scale)] for scale in (None, 0.3)]
        for rep in range(3):
            for g in graphs:
                g.replay()
            again = call(ws)
            graphs[rep % 2].replay()
            torch.cuda.synchronize()
            for got, first in zip(outs + [again], eager + eager[:1]):
                assert all(torch.equal(a, b) for a, b in zip(got, first))
            assert not ws[:65536].any()


@pytest.mark.parametrize("given", [False, True])
def test_outputs_belong_to_the_stream_that_writes_them(dev, given):
    rng = np.random.default_rng(39)
    D, T, lens, ps = 64, 9, [100, 30], 16
    c = E.Cache8(rng, dev, np.array(lens) + T, 2, ps, D)
    q, _ = R.rounded(rng, (2, 4, T, D), True, dev)
    rows, _ = R.rounded(rng, (2, 2, T, D), True, dev)
    par, kv = R.ints(R.tree(rng, 2, T), dev), R.ints(lens, dev)
    path, alen = R.ints([[0] + [-1] * (T - 1)] * 2, dev), R.ints([0, 0], dev)
    freq = dreams.rope_frequencies(D)
    k16 = torch.zeros((12, 2, ps, D), dtype=torch.bfloat16, device=dev)
    v16 = k16.clone()
    tab16 = R.ints(np.arange(12).reshape(2, 6) % 12, dev)
    kv16 = R.ints([3, 80], dev)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    kw = dict(stream=side) if given else {}
    with torch.cuda.stream(torch.cuda.current_stream() if given else side):
        got = [dreams.rope(q, freq, kv, **kw),
               dreams.paged_append_rope(rows, rows, k16, v16, tab16, kv16, freq, q=q, **kw),
               dreams.paged_append_e4m3(rows, rows, *c.pages, kv, frequencies=freq, q=q, parent=par, **kw),
               *dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=par, **kw),
               *dreams.paged_prompt_attn_e4m3(q, *c.pages, kv, **kw),
               dreams.paged_kv_commit_e4m3(*c.pages, kv, path, alen, **kw),
               *dreams.paged_read_e4m3(*c.pages, kv, 40, **kw)]
    torch.cuda.synchronize()
    for x in got:
        assert stream_of(x) == side.cuda_stream != stream_of(q)
