"""Attention over pages of 8 bits on the GPU against plain 64-bit definitions (tests/paged_ref.py) of the values that the codes
stand for.  Those values are exact in bf16, so the tolerances are the ones of bf16 pages."""
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


# heads, D, page, lengths, T, window, sinks, mask, paired, splits
VERIFY = [
    ((4, 4), 64, 16, [0], 1, 0, 0, False, False, 0),                     # one row, nothing but itself
    ((4, 4), 128, 16, [5, 0, 33], 1, 0, 0, False, False, 0),
    ((8, 2), 128, 16, [640], 16, 0, 0, False, False, 0),
    ((8, 2), 64, 32, [15, 16, 17, 31, 32, 33], 7, 0, 0, False, True, 0),  # ends at and around a block's and a step's
    ((16, 2), 128, 32, [47, 48, 49, 63, 64, 65], 3, 0, 0, False, True, 0),
    ((4, 1), 128, 16, [300, 77], 64, 0, 0, False, False, 0),
    ((7, 1), 128, 64, [511, 200], 65, 0, 0, False, False, 0),
    ((2, 2), 64, 128, [127, 1], 128, 0, 0, False, False, 0),
    ((14, 2), 128, 16, [1000], 100, 0, 0, False, True, 0),
    ((8, 8), 128, 256, [2000, 3, 900], 60, 0, 0, False, False, 0),
    ((8, 8), 64, 16, [2000, 1333], 33, 0, 0, False, False, 5),
    ((3, 3), 64, 32, [40, 0, 9], 17, 0, 0, True, False, 0),              # masks that leave rows empty
    ((8, 4), 128, 16, [0, 0], 70, 0, 0, True, False, 0),
    ((8, 2), 128, 16, [700, 90, 0], 1, 1, 0, False, False, 0),           # a window of the row alone
    ((8, 2), 128, 16, [700, 90, 3], 1, 64, 4, False, False, 0),
    ((8, 2), 64, 16, [700, 90, 0], 24, 3, 0, False, True, 0),            # a window shorter than the tree is deep
    ((8, 2), 128, 32, [700, 130, 10], 60, 100, 4, False, False, 0),
    ((4, 4), 128, 16, [700, 130, 10], 40, 97, 33, True, False, 0),
    ((4, 4), 64, 16, [500, 20], 128, 2, 600, False, False, 0),           # more sinks than slots
    ((4, 4), 128, 64, [1500, 1200], 9, 5000, 2, False, False, 0),        # a window longer than the cache
    ((8, 1), 128, 16, [1500, 1300], 60, 1024, 64, True, True, 4),
    ((16, 2), 128, 32, [2100], 128, 511, 1, False, False, 0),
    ((32, 32), 128, 64, [1000], 60, 0, 0, False, False, 0),
    ((8, 8), 64, 64, [5000, 4097], 1, 0, 0, False, False, 0),            # long: pieces
    ((32, 4), 64, 16, [3000], 4, 0, 0, False, False, 0),
]


@pytest.mark.parametrize("heads,D,ps,lens,T,window,sinks,masked,paired,splits", VERIFY)
def test_verify(dev, heads, D, ps, lens, T, window, sinks, masked, paired, splits):
    rng = np.random.default_rng(1)
    B, (Hq, Hkv) = len(lens), heads
    note("verify_e4m3", heads, D, ps, lens, T, window, sinks, masked, paired, splits)
    c = E.Cache8(rng, dev, np.array(lens) + T, Hkv, ps, D, paired)
    q, qh = R.rounded(rng, (B, Hq, T, D), True, dev)
    par = R.tree(rng, B, T)
    see = R.ancestors(par)
    if masked:
        see &= rng.random(see.shape) < 0.5
    mask = torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None
    want = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
    for bound in (0, max(1, max(lens))):
        out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), tree_mask=mask,
                                                 window=window, sinks=sinks, num_splits=splits,
                                                 max_kv_len=min(bound, max(1, c.width * ps - T)))
        R.check(out, lse, want, True, (heads, D, lens, T, bound))


# heads, D, page, lengths, rows, N, window, sinks, paired, splits
PROMPT = [
    ((4, 4), 64, 16, [0], [1], 1, 0, 0, False, 0),
    ((4, 2), 128, 16, [0, 0, 0], [5, 16, 1], 16, 0, 0, False, 0),
    ((8, 2), 64, 16, [0, 3, 40], [33, 0, 31], 33, 0, 0, True, 0),
    ((4, 4), 128, 32, [0, 0], [130, 7], 130, 0, 0, False, 0),
    ((28, 4), 128, 16, [17], [200], 200, 0, 0, False, 0),
    ((3, 1), 64, 64, [500, 1], [129, 128], 129, 0, 0, False, 0),
    ((8, 8), 128, 64, [0], [700], 700, 0, 0, False, 0),
    ((8, 2), 128, 16, [300, 20], [150, 90], 150, 64, 4, True, 0),
    ((4, 4), 64, 16, [0, 900], [257, 100], 257, 1, 0, False, 0),
    ((8, 1), 128, 32, [1000], [140], 140, 333, 33, False, 0),
    ((2, 2), 128, 16, [1000, 0], [60, 300], 300, 0, 0, False, 3),
    ((4, 1), 64, 256, [2000], [40], 40, 0, 0, False, 7),
    ((8, 2), 64, 16, [0, 100], [600, 555], 600, 100, 40, False, 0),
    ((4, 2), 128, 16, [31, 0], [0, 0], 9, 0, 0, False, 0),
]


@pytest.mark.parametrize("heads,D,ps,lens,rows,N,window,sinks,paired,splits", PROMPT)
def test_prompt(dev, heads, D, ps, lens, rows, N, window, sinks, paired, splits):
    rng = np.random.default_rng(2)
    B, (Hq, Hkv) = len(lens), heads
    note("prompt_e4m3", heads, D, ps, lens, rows, N, window, sinks, paired, splits)
    width = -(-(max(lens) + N) // ps)
    c = E.Cache8(rng, dev, np.array(lens) + rows, Hkv, ps, D, paired, width=width)
    q, qh = R.rounded(rng, (B, Hq, N, D), True, dev)
    for b in range(B):
        q[b, :, rows[b]:] = float("nan")        # rows past a prompt's own may hold anything
    want = R.prompt(qh, c.k, c.v, c.table, lens, rows, window, sinks, 1 / np.sqrt(D))
    for bound in (0, max(1, max(lens))):
        out, lse = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints(lens, dev), R.ints(rows, dev), window=window,
                                                 sinks=sinks, num_splits=splits,
                                                 max_kv_len=min(bound, max(1, c.width * ps - N)))
        R.check(out, lse, want, True, (heads, D, lens, rows, bound))


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,ps,lens,T", [((8, 2), 128, 16, [700, 333], 9), ((4, 4), 64, 32, [900], 16),
                                               ((8, 2), 128, 64, [800, 5], 60), ((2, 2), 128, 16, [1300], 100),
                                               ((16, 2), 64, 16, [450, 20], 70)])
def test_as_bf16_pages(dev, heads, D, ps, lens, T, kind):
    """The same values in bf16 pages: the calls differ by the order of their sums at most."""
    rng = np.random.default_rng(3)
    B, (Hq, Hkv) = len(lens), heads
    c = E.Cache8(rng, dev, np.array(lens) + T, Hkv, ps, D)
    k, v = (torch.from_numpy(np.nan_to_num(x, nan=3e38, posinf=3e38, neginf=-3e38)).to(torch.bfloat16).to(dev) for x in (c.k, c.v))
    for x, y in ((k, c.k), (v, c.v)):
        live = np.isfinite(y) & (np.abs(y) < 1e6)
        assert np.array_equal(x.double().cpu().numpy()[live], y[live])
    q, qh = R.rounded(rng, (B, Hq, T, D), True, dev)
    kv, par = R.ints(lens, dev), R.tree(rng, B, T)
    if kind == "verify":
        want = R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D))
        got = dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=R.ints(par, dev))
        other = dreams.paged_verify_attn(q, k, v, c.tabled, kv, parent=R.ints(par, dev))
    else:
        want = R.prompt(qh, c.k, c.v, c.table, lens, [T] * B, 0, 0, 1 / np.sqrt(D))
        got = dreams.paged_prompt_attn_e4m3(q, *c.pages, kv)
        other = dreams.paged_prompt_attn(q, k, v, c.tabled, kv)
    R.check(*got, want, True, "8 bits")
    R.check(*other, want, True, "16 bits")


@pytest.mark.parametrize("T,lens", [(1, [2100, 7]), (12, [900, 40]), (64, [900, 40]), (100, [640, 33])])
@pytest.mark.parametrize("scale", [0.3, -0.2, 0.0])
def test_scales_no_lse_and_large_blocks(dev, T, lens, scale):
    """Softmax scales of either sign, blocks whose scale bytes are far apart, no lse."""
    rng = np.random.default_rng(4)
    D, H, ps, B = 128, 2, 16, len(lens)
    c = E.Cache8(rng, dev, np.array(lens) + T, H, ps, D, scale=0.05)
    q, qh = R.rounded(rng, (B, 2 * H, T, D), True, dev)
    par = R.tree(rng, B, T)
    want = R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, scale)
    out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), scale=scale)
    R.check(out, lse, want, True, "scale")
    bare, none = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), scale=scale,
                                               with_lse=False)
    assert none is None and torch.equal(bare, out)


def test_lengths_and_parents_out_of_range(dev):
    """They are clamped, broken parents end a walk: finite results, no access outside the pool."""
    rng = np.random.default_rng(5)
    D, H, ps, T = 128, 2, 16, 10
    c = E.Cache8(rng, dev, [64, 64, 64], H, ps, D, width=4)
    q, _ = R.rounded(rng, (3, 4, T, D), True, dev)
    par = R.tree(rng, 3, T)
    par[0, 4], par[1, 2], par[2, 0] = 9, -7, 3
    got = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints([-5, 2 ** 31 - 1, 54], dev), parent=R.ints(par, dev))
    for x in got:
        assert torch.isfinite(x).all()
    got = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints([-5, 2 ** 31 - 1, 54], dev), R.ints([99, -3, T], dev))
    assert torch.isfinite(got[0]).all() and (got[0][1] == 0).all()


@pytest.mark.parametrize("T", [1, 5, 40, 128])
def test_replayed_and_on_another_stream(dev, T):
    rng = np.random.default_rng(6)
    D, Hq, H, ps, lens = 128, 8, 2, 16, [900, 50]
    c = E.Cache8(rng, dev, np.array(lens) + T, H, ps, D)
    q, qh = R.rounded(rng, (2, Hq, T, D), True, dev)
    par = R.tree(rng, 2, T)
    kv, pard = R.ints(lens, dev), R.ints(par, dev)
    run = lambda **kw: (*dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=pard, **kw),
                        *dreams.paged_prompt_attn_e4m3(q, *c.pages, kv, **kw))
    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for rep in range(3):
        q.normal_()
        kv.copy_(torch.tensor([900 - rep, 50 - 7 * rep], dtype=torch.int32))
        want = run()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_step_as_a_server_runs_it(dev):
    """A prompt and steps of drafts: rows rotated into pages of 8 bits, attended, their path compacted, a fork going its own
    way.  Checked against 64-bit attention over what the cache reads back as."""
    rng = np.random.default_rng(7)
    D, Hq, H, ps, P, B = 128, 8, 2, 16, 40, 2
    freq = dreams.rope_frequencies(D, 1e4)
    t = R.Tables(B, 12, P, ps)
    table, count, kv, ref = t.on(dev)
    k, v = (torch.zeros((P, H, ps, D), dtype=torch.uint8, device=dev).fill_(0x7f).view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.full((P, H, 1), 255, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu) for _ in range(2))
    pages = (k, v, ks, vs)

    def rows(N):
        new = lambda h: torch.from_numpy(rng.standard_normal((B, N, h, D))).to(torch.bfloat16).to(dev).transpose(1, 2)
        return new(Hq), new(H), new(H)

    def values():
        n = 12 * ps
        full = R.ints([n] * B, dev)
        return [x.double().cpu().numpy() for x in dreams.paged_read_e4m3(*pages, table, full, n)]

    lens = [0, 0]
    q, kn, vn = rows(37)
    live = [37, 0]
    dreams.pages_reserve(table, count, ref, R.ints(live, dev), ps)
    qr = dreams.paged_append_e4m3(kn, vn, *pages, table, kv, row_len=R.ints(live, dev), frequencies=freq, q=q)
    out, lse = dreams.paged_prompt_attn_e4m3(qr, *pages, table, kv, R.ints(live, dev))
    kh, vh = values()
    one = R.attend(qr[0].double().cpu().numpy(), kh[0][:, :37], vh[0][:, :37], np.tri(37, dtype=bool), 1 / np.sqrt(D))
    R.check(out[:1], lse[:1], [x[None] for x in one], True, "prompt")
    assert (out[1] == 0).all()
    kv.copy_(torch.tensor(live, dtype=torch.int32))
    assert dreams.pages_fork_e4m3(*pages, table, count, kv, ref, R.ints([0], dev), R.ints([1], dev)).tolist() == [1]
    lens = [37, 37]
    for step in range(4):
        T = [9, 1, 20, 5][step]
        par = R.tree(rng, B, T)
        dep, see = R.depths(par), R.ancestors(par)
        dreams.pages_reserve(table, count, ref, R.ints(np.array(lens) + T, dev), ps)
        q, kn, vn = rows(T)
        qr = dreams.paged_append_e4m3(kn, vn, *pages, table, kv, frequencies=freq, q=q, parent=R.ints(par, dev))
        out, lse = dreams.paged_verify_attn_e4m3(qr, *pages, table, kv, parent=R.ints(par, dev))
        kh, vh = values()
        ref64 = []
        for b in range(B):
            L = lens[b]
            vis = np.concatenate((np.ones((T, L), bool), see[b]), axis=1)
            ref64.append(R.attend(qr[b].double().cpu().numpy(), kh[b][:, :L + T], vh[b][:, :L + T], vis, 1 / np.sqrt(D)))
        R.check(out, lse, [np.stack(x) for x in zip(*ref64)], True, "step")
        # the rows that were cached are the rotated ones, to half a step of e4m3 of the block's scale
        want, size, far = E.rotate(kn.double().cpu().numpy(), np.array(lens)[:, None, None] + dep[:, None], freq.cpu().numpy(),
                                   1.0, False)
        for b in range(B):
            got = kh[b][:, lens[b]:lens[b] + T]
            near = np.abs(want[b]) * 2.0 ** -4 + 2.0 ** -9 * np.abs(got).max()     # (subnormal codes: 2^-10 of at most twice the largest)
            assert (np.abs(got - want[b]) <= near * (1 + 1e-6) + 1e-6).all()
        path, taken = np.full((B, T), -1, np.int32), np.zeros(B, np.int32)
        for b in range(B):
            i = int(rng.integers(T))
            taken[b] = dep[b, i]
            while i >= 0:
                path[b, dep[b, i]] = i
                i = int(par[b, i])
        before = [x.copy() for x in (kh, vh)]
        kv.copy_(dreams.paged_kv_commit_e4m3(*pages, table, kv, R.ints(path, dev), R.ints(taken, dev)))
        kh, vh = values()
        for b in range(B):
            for k0 in range(taken[b] + 1):
                for x, y in ((kh, before[0]), (vh, before[1])):
                    a, e = x[b][:, lens[b] + k0], y[b][:, lens[b] + path[b, k0]]
                    assert (np.abs(a - e) <= 2.0 ** -9 * np.abs(x[b][:, :lens[b] + T]).max() * 2.0 ** -8).all()
            lens[b] += int(taken[b]) + 1
        assert kv.tolist() == lens
        dreams.pages_release(table, count, kv, ref, R.ints([0, 1], dev), ps, trim=True)


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,lens,T,splits", [
    ((5, 5), 128, [300, 0, 77], 1, 0), ((5, 5), 64, [300, 0, 77], 60, 0), ((9, 9), 128, [1000], 40, 0), ((22, 11), 128, [900], 20, 3),
    ((3, 3), 64, [700, 650, 31], 110, 0), ((6, 3), 128, [500], 90, 0), ((10, 5), 64, [333, 400, 1], 128, 2),
    ((28, 4), 64, [200, 190, 5], 7, 0), ((28, 4), 64, [1200], 8, 3)])
def test_units_beside_the_dies(dev, heads, D, lens, T, splits, kind):
    """Sequences times KV heads that are no multiple of 8."""
    rng = np.random.default_rng(8)
    B, (Hq, Hkv) = len(lens), heads
    note("units_e4m3", heads, D, lens, T, splits, kind)
    c = E.Cache8(rng, dev, np.array(lens) + T, Hkv, 32, D)
    q, qh = R.rounded(rng, (B, Hq, T, D), True, dev)
    if kind == "verify":
        par = R.tree(rng, B, T)
        want = R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D))
        out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), num_splits=splits)
    else:
        want = R.prompt(qh, c.k, c.v, c.table, lens, [T] * B, 0, 0, 1 / np.sqrt(D))
        out, lse = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints(lens, dev), num_splits=splits)
    R.check(out, lse, want, True, (heads, D, lens, T, kind))


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,ps,lens,T,window,sinks,masked,splits", [
    ((8, 2), 128, 16, [2100, 300], 6, 0, 0, False, 1), ((8, 2), 64, 64, [2100, 3], 8, 0, 0, True, 2), ((3, 3), 128, 64, [1500], 17, 0, 0, False, 1),
    ((1, 1), 64, 16, [2500, 1100, 0], 32, 0, 0, False, 1), ((4, 1), 128, 32, [4100, 900], 7, 3000, 33, False, 1),
    ((4, 1), 128, 16, [4100, 30], 5, 1200, 2, True, 1), ((40, 40), 128, 64, [70, 40, 0, 12, 9, 31, 64], 19, 0, 0, False, 0),
    ((290, 290), 64, 16, [50], 30, 0, 0, True, 0)])
def test_two_rings_to_a_compute_unit(dev, heads, D, ps, lens, T, window, sinks, masked, splits, kind):
    """17 to 32 rows in long pieces, or of more heads than there are compute units: workgroups of 4 waves."""
    rng = np.random.default_rng(11)
    B, (Hq, Hkv) = len(lens), heads
    note("rings", heads, D, ps, lens, T, window, sinks, masked, splits, kind)
    c = E.Cache8(rng, dev, np.array(lens) + T, Hkv, ps, D)
    q, qh = R.rounded(rng, (B, Hq, T, D), True, dev)
    kw = dict(window=window, sinks=sinks, num_splits=splits)
    if kind == "verify":
        par = R.tree(rng, B, T)
        see = R.ancestors(par)
        if masked:
            see &= rng.random(see.shape) < 0.5
        mask = torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None
        want = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
        out, lse = dreams.paged_verify_attn_e4m3(q, *c.pages, R.ints(lens, dev), parent=R.ints(par, dev), tree_mask=mask, **kw)
    else:
        rows = [T if b != 1 else T // 2 for b in range(B)]
        want = R.prompt(qh, c.k, c.v, c.table, lens, rows, window, sinks, 1 / np.sqrt(D))
        out, lse = dreams.paged_prompt_attn_e4m3(q, *c.pages, R.ints(lens, dev), R.ints(rows, dev), **kw)
    R.check(out, lse, want, True, (heads, D, lens, T, kind))


def spread(q, c, **kw):
    """Whether the library spreads a call's keys in pieces of one length (its workspace has room for their rows alone)."""
    import ctypes
    desc, _ = dreams._paged_desc8(q, *c.pages, kw.get("window", 0), kw.get("sinks", 0), kw.get("max_kv_len", 0), 0, None)
    n, lib = ctypes.c_size_t(0), dreams.lib()
    size = lib.dreams_paged_prompt_attn_e4m3_workspace_size if kw.get("prompt") else lib.dreams_paged_verify_attn_e4m3_workspace_size
    assert size(ctypes.byref(desc), ctypes.byref(n)) == 0
    rows = desc.num_q_heads // desc.num_kv_heads * desc.num_rows
    rows = 16 if rows <= 16 else 32 if rows <= 32 else 64
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    wgs = max(2 * cus if rows == 64 else cus, 2 * desc.batch * desc.num_kv_heads)
    return n.value == dreams.WORKSPACE_COUNTER_BYTES + wgs * rows * (desc.head_dim * 4 + 8)


# heads, D, lengths, T, window, sinks, mask
SPREAD = [
    ((4, 1), 128, [8000, 10, 3333], 1, 0, 0, False),
    ((7, 1), 128, [6100, 0, 5, 2048, 700], 4, 0, 0, False),
    ((2, 1), 64, [15000], 1, 0, 0, False),
    ((3, 1), 64, [6500, 4095, 1], 5, 0, 0, True),
    ((4, 1), 128, [6200, 4100, 900], 14, 0, 0, False),
    ((16, 2), 128, [3900, 17, 8000], 2, 0, 0, False),
    ((2, 1), 128, [9000, 300, 8000], 9, 7000, 40, False),
    ((4, 1), 128, [20000, 10, 3333], 1, 0, 0, False),          # from here on they are spread
    ((3, 1), 64, [20100, 4095, 1], 5, 0, 0, True),
    ((4, 1), 128, [20200, 0, 900], 14, 0, 0, False),
    ((16, 2), 128, [17000], 2, 0, 0, False),
    ((2, 1), 128, [21000, 300, 8000], 9, 19700, 40, False),
]


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,lens,T,window,sinks,masked", SPREAD)
def test_long_keys_of_few_heads(dev, heads, D, lens, T, window, sinks, masked, kind):
    """Pieces of one length over every sequence and a second launch that merges them; twice the same, bit for bit."""
    rng = np.random.default_rng(9)
    B, (Hq, Hkv), ps = len(lens), heads, 64
    note("spread", heads, D, lens, T, window, sinks, masked, kind)
    c = E.Cache8(rng, dev, np.array(lens) + T, Hkv, ps, D)
    q, qh = R.rounded(rng, (B, Hq, T, D), True, dev)
    kw = dict(window=window, sinks=sinks, max_kv_len=max(lens))
    assert spread(q, c, prompt=kind == "prompt", **kw) or max(lens) < 17000
    kv = R.ints(lens, dev)
    if kind == "verify":
        par = R.tree(rng, B, T)
        see = R.ancestors(par)
        if masked:
            see &= rng.random(see.shape) < 0.5
        mask = torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None
        want = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
        run = lambda: dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=R.ints(par, dev), tree_mask=mask, **kw)
    else:
        rows = [T if b != 1 else 0 for b in range(B)]       # (a sequence without rows: zeros)
        rl = R.ints(rows, dev)
        want = R.prompt(qh, c.k, c.v, c.table, lens, rows, window, sinks, 1 / np.sqrt(D))
        run = lambda: dreams.paged_prompt_attn_e4m3(q, *c.pages, kv, rl, **kw)
    out, lse = run()
    R.check(out, lse, want, True, (heads, lens, kind))
    again = run()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("longest", [7198, 20198])
def test_long_keys_replayed(dev, longest):
    """Lengths that change between replays change the pieces."""
    rng = np.random.default_rng(10)
    D, ps, B, T = 128, 16, 3, 2
    c = E.Cache8(rng, dev, [longest + T] * 3, 1, ps, D)
    q, qh = R.rounded(rng, (B, 4, T, D), True, dev)
    par = R.tree(rng, B, T)
    kv, pard = R.ints([4000, 4000, 4000], dev), R.ints(par, dev)
    assert spread(q, c, max_kv_len=longest) or longest < 17000
    run = lambda: dreams.paged_verify_attn_e4m3(q, *c.pages, kv, parent=pard, max_kv_len=longest)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for lens in ([longest, 1, 300], [0, 0, 0], [31, 4100, 2500]):
        kv.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        R.check(*got, R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D)), True, lens)
        assert all(torch.equal(a, b) for a, b in zip(got, run()))
