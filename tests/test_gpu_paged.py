"""The paged cache's operators on the GPU against plain 64-bit definitions (tests/paged_ref.py)."""
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


# heads, D, page, lengths, T, window, sinks, mask, paired, splits
VERIFY = [
    ((4, 4), 64, 16, [0], 1, 0, 0, False, False, 0),                     # one row, nothing but itself
    ((4, 4), 128, 16, [5, 0, 33], 1, 0, 0, False, False, 0),
    ((8, 2), 128, 16, [640], 16, 0, 0, False, False, 0),
    ((8, 2), 64, 32, [15, 16, 17, 31, 32, 33], 7, 0, 0, False, True, 0),  # ends at and around a page's and a step's
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
    ((8, 1), 128, 16, [3000, 2500], 60, 1024, 64, True, True, 4),
    ((16, 2), 128, 32, [4100], 128, 511, 1, False, False, 0),
    ((32, 32), 128, 64, [3136], 60, 0, 0, False, False, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,D,ps,lens,T,window,sinks,masked,paired,splits", VERIFY)
def test_verify(dev, heads, D, ps, lens, T, window, sinks, masked, paired, splits, dtype):
    if dtype == "f32" and max(lens) * heads[0] * T > 3e6:
        lens, T = [min(n, 900) for n in lens], min(T, 60)
    rng = np.random.default_rng(1)
    bf16, B = dtype == "bf16", len(lens)
    Hq, Hkv = heads
    note("verify", dtype, heads, D, ps, lens, T, window, sinks, masked, paired, splits)
    c = R.Cache(rng, dev, np.array(lens) + T, Hkv, ps, D, bf16, paired)
    q, qh = R.rounded(rng, (B, Hq, T, D), bf16, dev)
    par = R.tree(rng, B, T)
    see = R.ancestors(par)
    if masked:
        see &= rng.random(see.shape) < 0.5
        see[:, 0] = False
    out, lse = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), parent=R.ints(par, dev),
                                        tree_mask=torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None,
                                        window=window, sinks=sinks, num_splits=splits)
    torch.cuda.synchronize()
    ref = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
    note("  max error %.2e" % R.check(out, lse, ref, bf16, "verify"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 0.5])
def test_verify_scales_mask_alone_and_no_lse(dev, dtype, scale):
    rng = np.random.default_rng(2)
    bf16, D, T, lens = dtype == "bf16", 128, 20, [130, 47]
    c = R.Cache(rng, dev, np.array(lens) + T, 2, 16, D, bf16)
    q, qh = R.rounded(rng, (2, 6, T, D), bf16, dev)
    par = R.tree(rng, 2, T)
    see = R.ancestors(par)
    out, lse = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), scale=scale, with_lse=False,
                                        tree_mask=torch.from_numpy(R.mask_bits(see)).to(dev))
    assert lse is None
    R.check(out, None, R.verify(qh, c.k, c.v, c.table, lens, par, see, 0, 0, np.float64(np.float32(scale))), bf16, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_large_scores(dev, dtype):
    """Scores of several hundred, so that the running maximum moves and most weights vanish."""
    rng = np.random.default_rng(3)
    bf16, D, T, lens = dtype == "bf16", 64, 30, [700, 260]
    c = R.Cache(rng, dev, np.array(lens) + T, 2, 32, D, bf16, scale=8.0)
    q, qh = R.rounded(rng, (2, 4, T, D), bf16, dev, std=8.0)
    par = R.tree(rng, 2, T)
    out, lse = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), parent=R.ints(par, dev), window=300,
                                        sinks=2)
    R.check(out, lse, R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 300, 2, 1 / 8), bf16, "large")


def test_verify_takes_lengths_and_parents_out_of_range(dev):
    """kv_len is clamped, a parent that breaks the rules ends the walk; nothing is read outside the pool."""
    rng = np.random.default_rng(4)
    D, T, ps = 128, 6, 16
    c = R.Cache(rng, dev, [64, 64], 2, ps, D, True)
    q, qh = R.rounded(rng, (2, 2, T, D), True, dev)
    par = np.array([[-1, 0, 1, 3, 9, 2], [-1, -7, 0, 1, 2, 3]], np.int32)
    out, lse = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints([1000, -5], dev), parent=R.ints(par, dev))
    lens = [64 - T, 0]
    R.check(out, lse, R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D)), True, "clamped")


# heads, D, page, lengths, rows, N, window, sinks, paired, splits
PROMPT = [
    ((4, 4), 64, 16, [0], [1], 1, 0, 0, False, 0),
    ((4, 2), 128, 16, [0, 7], [5, 0], 5, 0, 0, False, 0),                # a sequence without rows
    ((8, 2), 128, 32, [0, 0, 0], [63, 64, 65], 65, 0, 0, False, 0),
    ((4, 1), 64, 16, [3, 40], [130, 127], 130, 0, 0, True, 0),
    ((6, 2), 128, 16, [0], [257], 257, 0, 0, False, 0),
    ((8, 2), 128, 64, [100, 0, 31], [300, 17, 288], 300, 0, 0, False, 0),
    ((2, 2), 128, 16, [900], [40], 40, 0, 0, False, 0),                  # few rows behind a long prefix
    ((2, 1), 64, 32, [2100, 1700], [200, 150], 200, 0, 0, False, 0),
    ((8, 8), 128, 128, [0], [700], 700, 0, 0, False, 0),
    ((4, 2), 128, 16, [0, 200], [300, 211], 300, 1, 0, False, 0),        # every row alone
    ((4, 2), 128, 16, [0, 200], [300, 211], 300, 16, 4, False, 0),
    ((4, 2), 64, 32, [50, 700], [400, 333], 400, 100, 70, True, 0),
    ((4, 4), 128, 16, [600], [300], 300, 257, 0, False, 0),
    ((4, 4), 64, 16, [20], [290], 290, 40, 400, False, 0),               # more sinks than slots
    ((2, 2), 128, 64, [1000], [520], 520, 4000, 3, False, 0),
    ((2, 2), 128, 32, [1500, 40], [129, 1], 129, 600, 5, False, 3),
    ((4, 1), 128, 16, [1500], [260], 260, 0, 0, False, 4),
    ((7, 1), 64, 256, [0], [1030], 1030, 0, 0, False, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,D,ps,lens,rows,N,window,sinks,paired,splits", PROMPT)
def test_prompt(dev, heads, D, ps, lens, rows, N, window, sinks, paired, splits, dtype):
    rng = np.random.default_rng(5)
    bf16, B = dtype == "bf16", len(lens)
    Hq, Hkv = heads
    note("prompt", dtype, heads, D, ps, lens, rows, N, window, sinks, paired, splits)
    width = -(-(max(lens) + N) // ps)
    c = R.Cache(rng, dev, np.array(lens) + np.array(rows), Hkv, ps, D, bf16, paired, width=width)
    q, qh = R.rounded(rng, (B, Hq, N, D), bf16, dev)
    q[:, :, max(rows):] = float("nan")
    for b in range(B):
        q[b, :, rows[b]:] = float("nan")      # rows behind a sequence's last
        qh[b, :, rows[b]:] = 0
    out, lse = dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), R.ints(rows, dev), window=window,
                                        sinks=sinks, num_splits=splits)
    torch.cuda.synchronize()
    ref = R.prompt(qh, c.k, c.v, c.table, lens, rows, window, sinks, 1 / np.sqrt(D))
    note("  max error %.2e" % R.check(out, lse, ref, bf16, "prompt"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [40, 200])
def test_prompt_defaults_and_ranges(dev, dtype, N):
    """No row_len: all rows; lengths and row counts out of range are clamped; a negative scale, no lse."""
    rng = np.random.default_rng(6)
    bf16, D, ps = dtype == "bf16", 128, 16
    c = R.Cache(rng, dev, [304, 304], 2, ps, D, bf16)
    q, qh = R.rounded(rng, (2, 4, N, D), bf16, dev)
    out, lse = dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, R.ints([9999, -3], dev), scale=-0.3, with_lse=False)
    ref = R.prompt(qh, c.k, c.v, c.table, [304 - N, 0], [N, N], 0, 0, np.float64(np.float32(-0.3)))
    assert lse is None
    R.check(out, None, ref, bf16, "all rows")
    out, lse = dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, R.ints([5, 5], dev), R.ints([-4, 9999], dev))
    R.check(out, lse, R.prompt(qh, c.k, c.v, c.table, [5, 5], [0, N], 0, 0, 1 / np.sqrt(D)), bf16, "row counts")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_pool_past_32_bits(dev, dtype):
    """Pages more than 2^32 bytes into a pool, and page numbers times page sizes past 2^31 elements."""
    bf16, D, ps, Hkv, T = dtype == "bf16", 128, 16, 1, 5
    rng = np.random.default_rng(7)
    dt = torch.bfloat16 if bf16 else torch.float32
    size = 2 if bf16 else 4
    P = (1 << 32) * 5 // 4 // (ps * D * size)
    k = torch.empty((P, Hkv, ps, D), dtype=dt, device=dev)
    v = torch.empty((P, Hkv, ps, D), dtype=dt, device=dev)
    lens, rows = [70], 21
    table = np.array([[P - 1, 3, P - 9, P // 2, P - 2, 1, P - 77, 0]], np.int32)
    new_k, kh = R.rounded(rng, (1, Hkv, 100, D), bf16, dev)
    new_v, vh = R.rounded(rng, (1, Hkv, 100, D), bf16, dev)
    tab = R.ints(table, dev)
    dreams.paged_append(new_k, new_v, k, v, tab, R.ints([0], dev))
    slots_k, slots_v = np.zeros((8, Hkv, ps, D)), np.zeros((8, Hkv, ps, D))
    for j in range(100):
        slots_k[j // ps, :, j % ps], slots_v[j // ps, :, j % ps] = kh[0, :, j], vh[0, :, j]
    near = np.arange(8, dtype=np.int32)[None]
    q, qh = R.rounded(rng, (1, 2, T, D), bf16, dev)
    par = R.tree(rng, 1, T)
    out, lse = dreams.paged_verify_attn(q, k, v, tab, R.ints(lens, dev), parent=R.ints(par, dev))
    R.check(out, lse, R.verify(qh, slots_k, slots_v, near, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D)), bf16, "far")
    q, qh = R.rounded(rng, (1, 2, rows, D), bf16, dev)
    out, lse = dreams.paged_prompt_attn(q, k, v, tab, R.ints(lens, dev), R.ints([rows], dev))
    R.check(out, lse, R.prompt(qh, slots_k, slots_v, near, lens, [rows], 0, 0, 1 / np.sqrt(D)), bf16, "far prompt")
    for t in (k, v):
        assert torch.equal(t[P - 1], (new_k if t is k else new_v)[0, :, :ps])
    # a move between far pages, and a fork of a far, partly filled page
    kept = dreams.paged_kv_commit(k, v, tab, R.ints([60], dev), R.ints([[0, 30]], dev), R.ints([1], dev))
    assert kept.tolist() == [62]
    assert torch.equal(k[int(table[0, 61 // ps]), :, 61 % ps], new_k[0, :, 90])
    tab2 = torch.cat((tab, torch.full_like(tab, -1)))
    if P <= dreams.PAGES_MAX:
        ref = torch.ones(P, dtype=torch.int32, device=dev)
        ref[P - 5] = 0
        cnt, ln = R.ints([7, 0], dev), R.ints([100, 0], dev)
        g = dreams.pages_fork(k, v, tab2, cnt, ln, ref, R.ints([0], dev), R.ints([1], dev))
        assert g.tolist() == [1] and tab2[1].tolist()[:7] == table[0].tolist()[:6] + [P - 5]
        assert torch.equal(k[P - 5, :, :4], new_k[0, :, 96:100])


# ------------------------------------------------------------------------------------------------------------- rows
def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


def random_bits(rng, shape, dt, dev):
    n = np.int16 if dt == torch.bfloat16 else np.int32
    info = np.iinfo(n)
    return torch.from_numpy(rng.integers(info.min, info.max, size=shape, dtype=n, endpoint=True)).to(dev).view(dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("NL,Hkv,ps,D,lens,N,rows,order,paired", [
    (1, 1, 16, 64, [0], 1, None, "heads", False),
    (3, 2, 16, 128, [15, 0, 40], 20, [20, 3, 0], "tokens", False),
    (2, 4, 32, 64, [31, 33], 70, None, "tokens", True),
    (1, 3, 64, 8, [5, 60, 0, 7], 9, [9, 20, -1, 1], "heads", False),
    (2, 8, 16, 128, [100], 128, None, "strided", True),
])
def test_append(dev, dt, NL, Hkv, ps, D, lens, N, rows, order, paired):
    rng = np.random.default_rng(8)
    B = len(lens)
    counts = -(-(np.array(lens) + N) // ps)
    P, width = int(counts.sum()) + 2, int(counts.max())
    ids = rng.permutation(P).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :counts[b]] = ids[at:at + counts[b]]
        at += counts[b]
    if B > 1:
        table[0, counts[0] - 1] = P + 5      # a page outside the pool: its rows are left out
    if paired:
        both = random_bits(rng, (NL, P, 2, Hkv, ps, D), dt, dev)
        k, v = both[:, :, 0], both[:, :, 1]
    else:
        k, v = random_bits(rng, (NL, P, Hkv, ps, D), dt, dev), random_bits(rng, (NL, P, Hkv, ps, D), dt, dev)
    shape = {"heads": (NL, B, Hkv, N, D), "tokens": (NL, B, N, Hkv, D), "strided": (NL, B, Hkv, 2 * N, 2 * D)}[order]
    new = [random_bits(rng, shape, dt, dev) for _ in range(2)]
    if order == "tokens":
        new = [x.transpose(2, 3) for x in new]
    if order == "strided":
        new = [x[:, :, :, 1::2, D:] for x in new]
    want = [bits(k).copy(), bits(v).copy()]
    for w, x in zip(want, new):
        xb = bits(x)
        for b in range(B):
            for i in range(N if rows is None else min(max(rows[b], 0), N)):
                j = lens[b] + i
                page = table[b, j // ps]
                if 0 <= page < P:
                    w[:, page, :, j % ps] = xb[:, b, :, i]
    dreams.paged_append(new[0], new[1], k, v, R.ints(table, dev), R.ints(lens, dev),
                        None if rows is None else R.ints(rows, dev))
    torch.cuda.synchronize()
    assert np.array_equal(bits(k), want[0]) and np.array_equal(bits(v), want[1])
    # one layer's pools without the layer axis; nothing to write for a negative length or past the table
    before = bits(k).copy()
    dreams.paged_append(new[0][0], new[1][0], k[0], v[0], R.ints(table, dev), R.ints([-1] * B, dev))
    dreams.paged_append(new[0][0], new[1][0], k[0], v[0], R.ints(table, dev), R.ints([width * ps] * B, dev))
    dreams.paged_append(new[0][0], new[1][0], k[0], v[0], R.ints(table, dev), R.ints([2 ** 31 - 1] * B, dev))
    assert np.array_equal(bits(k), before)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("paired", [False, True])
def test_commit(dev, dt, paired):
    rng = np.random.default_rng(9)
    NL, Hkv, ps, D, T = 3, 2, 16, 128, 100
    paths = [[0, 2, 5, 7], [0], [0, 1, 4], [0, 2, 3, 5, 6, 8], list(range(0, 100, 2)), [0, 60, 61]]
    lens = [10, 0, 31, 54, 12, 40]
    B = len(paths)
    counts = -(-(np.array(lens) + T) // ps)
    counts[5] = 5                       # its last sources lie past the table
    P, width = int(counts.sum()) + 1, int(counts.max())
    ids = rng.permutation(P).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :counts[b]] = ids[at:at + counts[b]]
        at += counts[b]
    if paired:
        both = random_bits(rng, (NL, P, 2, Hkv, ps, D), dt, dev)
        k, v = both[:, :, 0], both[:, :, 1]
    else:
        k, v = random_bits(rng, (NL, P, Hkv, ps, D), dt, dev), random_bits(rng, (NL, P, Hkv, ps, D), dt, dev)
    path = np.full((B, T), -1, np.int32)
    alen = np.array([len(p) - 1 for p in paths], np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    want = [bits(k).copy(), bits(v).copy()]
    for w in want:
        for b in range(B):
            for n in range(alen[b] + 1):
                s, t = lens[b] + path[b, n], lens[b] + n
                if path[b, n] > n and s // ps < counts[b]:
                    w[:, table[b, t // ps], :, t % ps] = w[:, table[b, s // ps], :, s % ps]
    out = dreams.paged_kv_commit(k, v, R.ints(table, dev), R.ints(lens, dev), R.ints(path, dev), R.ints(alen, dev))
    torch.cuda.synchronize()
    assert out.tolist() == [n + a + 1 for n, a in zip(lens, alen)]
    assert np.array_equal(bits(k), want[0]) and np.array_equal(bits(v), want[1])


# ------------------------------------------------------------------------------------------------------------ tables
@pytest.mark.parametrize("B,width,P,ps", [(1, 1, 1, 16), (5, 9, 40, 16), (40, 30, 700, 32), (3, 4, 64, 16), (3, 4, 65, 16),
                                          (300, 12, 2500, 16), (4, 5000, 130000, 16)])
def test_reserve_and_release(dev, B, width, P, ps):
    rng = np.random.default_rng(B + P)
    t = R.Tables(B, width, P, ps)
    held = rng.random(P) < 0.3
    t.ref[held] = rng.integers(1, 4, size=int(held.sum()))     # pages that others hold
    on = t.on(dev)
    table, count, kv_len, ref = on
    for step in range(6):
        want = rng.integers(-5, width * ps + 40, size=B).astype(np.int32)
        if step % 2:
            want = (t.count * ps + rng.integers(0, 40, size=B)).astype(np.int32)
        got = dreams.pages_reserve(table, count, ref, R.ints(want, dev), ps)
        assert got.tolist() == t.reserve(want), step
        t.same(on)
        t.kv_len[:] = np.minimum(np.maximum(want, 0), t.count * ps)
        kv_len.copy_(R.ints(t.kv_len, dev))
        seqs = rng.integers(-2, B + 2, size=max(1, B // 2))
        trim = step % 3 == 1
        dreams.pages_release(table, count, kv_len, ref, R.ints(seqs, dev), ps, trim=trim)
        t.release(seqs, trim)
        t.same(on)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("NL,Hkv,ps,D,B,spare,paired", [(1, 1, 16, 64, 3, 2, False), (2, 3, 16, 128, 9, 1, True),
                                                         (3, 2, 64, 128, 20, 4, False), (1, 1, 1024, 128, 6, 9, True)])
def test_fork(dev, dt, NL, Hkv, ps, D, B, spare, paired):
    rng = np.random.default_rng(B)
    width = 7
    t = R.Tables(B, width, B * 4 + spare, ps)
    P = len(t.ref)
    lens = rng.integers(0, 4 * ps, size=B).astype(np.int32)
    lens[0], lens[1] = 2 * ps, 3 * ps - 1
    lens[B // 2:] = 0
    t.reserve(lens)
    t.kv_len[:] = lens
    t.ref[rng.choice(t.free(), size=max(0, len(t.free()) - spare - 1), replace=False)] = 1    # a nearly full pool
    if paired:
        both = random_bits(rng, (NL, P, 2, Hkv, ps, D), dt, dev)
        k, v = both[:, :, 0], both[:, :, 1]
    else:
        k, v = random_bits(rng, (NL, P, Hkv, ps, D), dt, dev), random_bits(rng, (NL, P, Hkv, ps, D), dt, dev)
    on = t.on(dev)
    table, count, kv_len, ref = on
    # copies of the first sequences; a copy named twice, one that holds pages, itself, indices outside, a source that becomes a
    # copy in the same call
    src = [1, 0, 1, 0, -1, 1, B, B - 1] + [int(x) for x in rng.integers(0, B, size=B)]
    dst = [B - 1, B - 1, 0, 0, B - 1, B, B - 2, B - 2] + [int(x) for x in rng.integers(0, B, size=B)]
    want = [bits(k).copy(), bits(v).copy()]
    granted, copies = t.fork(src, dst)
    for w in want:
        for a, b, n in copies:
            w[:, b, :, :n] = w[:, a, :, :n]
    got = dreams.pages_fork(k, v, table, count, kv_len, ref, R.ints(src, dev), R.ints(dst, dev))
    assert got.tolist() == granted
    t.same(on)
    assert np.array_equal(bits(k), want[0]) and np.array_equal(bits(v), want[1])
    dreams.pages_release(table, count, kv_len, ref, R.ints(list(range(B)), dev), ps)
    t.release(range(B))
    t.same(on)


def test_fork_of_a_sequence_whose_pages_do_not_cover_it(dev):
    t = R.Tables(3, 4, 8, 16)
    t.reserve([20, 0, 0])
    t.kv_len[:] = [40, 0, 0]
    on = t.on(dev)
    k = torch.zeros((8, 1, 16, 64), device=dev)
    got = dreams.pages_fork(k, k.clone(), *on[:2], on[2], on[3], R.ints([0], dev), R.ints([1], dev))
    assert got.tolist() == [0]
    t.same(on)
    t.kv_len[0] = -1
    on[2].copy_(R.ints(t.kv_len, dev))
    assert dreams.pages_fork(k, k.clone(), *on[:2], on[2], on[3], R.ints([0], dev), R.ints([1], dev)).tolist() == [0]
    t.same(on)


# ---------------------------------------------------------------------------------------------- a run of them together
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 3)])
def test_prompts_steps_and_forks(dev, dt, window, sinks):
    """Two prompts in pieces, verify steps with acceptance and commit, a fork whose branches go on apart, a release: every
    attention call against the definition over the rows that were written, kept by hand."""
    rng = np.random.default_rng(10)
    bf16 = dt == torch.bfloat16
    B, Hq, Hkv, D, ps, P, width, T, NL = 4, 4, 2, 64, 16, 60, 20, 12, 2
    table, count, kv_len, ref = R.Tables(B, width, P, ps).on(dev)
    k = torch.full((NL, P, Hkv, ps, D), float("nan"), dtype=dt, device=dev)
    v = torch.full((NL, P, Hkv, ps, D), float("nan"), dtype=dt, device=dev)
    kept = [[np.zeros((NL, Hkv, 0, D)) for _ in range(2)] for _ in range(B)]     # K and V rows of every sequence
    scale = 1 / np.sqrt(D)

    def dense(b, layer, extra):
        """A pool of one page that holds a sequence's rows and the given new ones."""
        return [np.concatenate((kept[b][i][layer], extra[i][layer, b]), axis=1)[None] for i in range(2)]

    def prompt_piece(N, rows):
        nonlocal kv_len
        rows = np.array(rows)
        (kn, kh), (vn, vh) = (R.rounded(rng, (NL, B, N, Hkv, D), bf16, dev) for _ in range(2))
        kh, vh = kh.transpose(0, 1, 3, 2, 4), vh.transpose(0, 1, 3, 2, 4)
        assert dreams.pages_reserve(table, count, ref, kv_len + R.ints(rows, dev), ps).tolist() == [1] * B
        dreams.paged_append(kn.transpose(2, 3), vn.transpose(2, 3), k, v, table, kv_len, R.ints(rows, dev))
        for layer in range(NL):
            q, qh = R.rounded(rng, (B, Hq, N, D), bf16, dev)
            out, lse = dreams.paged_prompt_attn(q, k[layer], v[layer], table, kv_len, R.ints(rows, dev), window, sinks)
            for b in range(B):
                L = kept[b][0].shape[2]
                kk, vv = dense(b, layer, (kh[:, :, :, :rows[b]], vh[:, :, :, :rows[b]]))
                ref64 = R.prompt(qh[b:b + 1], kk, vv, np.zeros((1, 1), np.int32), [L], [rows[b]], window, sinks, scale)
                R.check(out[b:b + 1], lse[b:b + 1], ref64, bf16, ("prompt", layer, b))
        for b in range(B):
            kept[b] = [np.concatenate((x, n[:, b, :, :rows[b]]), axis=2) for x, n in zip(kept[b], (kh, vh))]
        kv_len = kv_len + R.ints(rows, dev)

    def step(active):
        nonlocal kv_len
        par = R.tree(rng, B, T, 4, 3)
        (kn, kh), (vn, vh) = (R.rounded(rng, (NL, B, Hkv, T, D), bf16, dev) for _ in range(2))
        on = np.array([b in active for b in range(B)])
        want = torch.where(torch.from_numpy(on).to(dev), kv_len + T, torch.zeros_like(kv_len))
        assert dreams.pages_reserve(table, count, ref, want, ps).tolist() == [1] * B
        dreams.paged_append(kn, vn, k, v, table, kv_len, R.ints(T * on, dev))
        for layer in range(NL):
            q, qh = R.rounded(rng, (B, Hq, T, D), bf16, dev)
            out, lse = dreams.paged_verify_attn(q, k[layer], v[layer], table, kv_len, R.ints(par, dev), window=window,
                                                sinks=sinks)
            for b in active:
                L = kept[b][0].shape[2]
                kk, vv = dense(b, layer, (kh, vh))
                ref64 = R.verify(qh[b:b + 1], kk, vv, np.zeros((1, 1), np.int32), [L], par[b:b + 1],
                                 R.ancestors(par[b:b + 1]), window, sinks, scale)
                R.check(out[b:b + 1], lse[b:b + 1], ref64, bf16, ("verify", layer, b))
        logits = rng.standard_normal((B, T, 50)).astype(np.float32)
        am = logits.argmax(2)
        tok = np.where(rng.random((B, T)) < 0.7, np.take_along_axis(am, np.maximum(par, 0).astype(np.int64), 1), 0)
        alen, path, _, _ = dreams.tree_accept(torch.from_numpy(logits).to(dev), R.ints(tok, dev), R.ints(par, dev))
        after = dreams.paged_kv_commit(k, v, table, kv_len, path, alen)
        path, alen = path.cpu().numpy(), alen.cpu().numpy()
        for b in active:
            way = path[b, :alen[b] + 1]
            kept[b] = [np.concatenate((x, n[:, b][:, :, way]), axis=2) for x, n in zip(kept[b], (kh, vh))]
        kv_len = torch.where(torch.from_numpy(on).to(dev), after, kv_len)
        assert kv_len.tolist() == [x[0].shape[2] for x in kept]

    prompt_piece(40, [40, 23, 0, 0])
    prompt_piece(30, [7, 30, 0, 0])
    step([0, 1])
    step([0, 1])
    got = dreams.pages_fork(k, v, table, count, kv_len, ref, R.ints([0, 1], dev), R.ints([3, 2], dev))
    assert got.tolist() == [1, 1]
    kept[3], kept[2] = [x.copy() for x in kept[0]], [x.copy() for x in kept[1]]
    for _ in range(3):
        step([0, 1, 2, 3])          # the branches go apart
    dreams.pages_release(table, count, kv_len, ref, R.ints([0], dev), ps)
    kept[0] = [np.zeros((NL, Hkv, 0, D)) for _ in range(2)]
    step([1, 2, 3])
    prompt_piece(50, [50, 1, 0, 20])   # another prompt in the pages that came free
    step([0, 1, 2, 3])
    dreams.pages_release(table, count, kv_len, ref, R.ints([0, 1, 2, 3], dev), ps, trim=True)
    held = -(-kv_len.cpu().numpy() // ps)
    assert count.cpu().numpy().tolist() == held.tolist()
    dreams.pages_release(table, count, kv_len, ref, R.ints([3, 2, 1, 0, 0], dev), ps)
    assert int(ref.abs().sum()) == 0 and int(count.sum()) == 0 and int(kv_len.sum()) == 0 and int((table != -1).sum()) == 0


# -------------------------------------------------------------------------------- graphs, streams, workspaces, waits
def attention_case(rng, dev, dt, kind):
    bf16 = dt == torch.bfloat16
    Hq, Hkv, D, ps, lens = 8, 2, 128, 16, [2100, 700]
    T = 60 if kind == "verify" else 20 if kind == "verify16" else 200
    c = R.Cache(rng, dev, np.array(lens) + T, Hkv, ps, D, bf16)
    q, _ = R.rounded(rng, (2, Hq, T, D), bf16, dev)
    kv = R.ints(lens, dev)
    if kind == "prompt":
        rows = R.ints([200, 77], dev)
        return lambda **kw: dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, kv, rows, window=900, sinks=3, **kw)
    par = R.ints(R.tree(rng, 2, T), dev)
    return lambda **kw: dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, kv, par, **kw)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["verify", "verify16", "prompt"])
def test_attention_replayed(dev, dt, kind):
    """Captured calls without a workspace of the caller's have their own: two graphs and eager calls do not share one."""
    call = attention_case(np.random.default_rng(11), dev, dt, kind)
    eager = [bits(t) for t in call(num_splits=4)]
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(num_splits=4))
        graphs.append(g)
    side = [torch.cuda.Stream() for _ in range(2)]
    filler = torch.zeros(333, device=dev)
    for rep in range(4):
        for pair in outs:
            for t in pair:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for g, s in zip(graphs, side):       # both at once
            with torch.cuda.stream(s):
                g.replay()
        filler.add_(1.0)
        other = call(num_splits=4)           # and an eager one
        torch.cuda.synchronize()
        for pair in outs + [other]:
            for t, want in zip(pair, eager):
                assert np.array_equal(bits(t), want), (kind, rep)


@pytest.mark.parametrize("kind", ["verify", "prompt"])
def test_attention_on_other_streams(dev, kind):
    call = attention_case(np.random.default_rng(12), dev, torch.bfloat16, kind)
    want = [bits(t) for t in call(num_splits=3)]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(3)]
    results = []
    for s in side:                           # as the current stream, one workspace each
        with torch.cuda.stream(s):
            results.append(call(num_splits=3))
    for s in side:                           # and given
        results.append(call(num_splits=3, stream=s))
    torch.cuda.synchronize()
    for r in results:
        for t, w in zip(r, want):
            assert np.array_equal(bits(t), w)
    outs = [torch.empty_like(results[0][0]), torch.empty_like(results[0][1])]
    with pytest.raises(ValueError, match="out must be"):
        call(out=outs[0][:, :1].contiguous())
    with pytest.raises(ValueError, match="workspace"):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(num_splits=3, stream=side[0])


def test_workspaces(dev):
    """A caller's workspace: too small is refused, left zero, free of flags; a wait that gives up is reported."""
    rng = np.random.default_rng(13)
    D, T, lens = 128, 60, [2000, 1900]
    for Hq, Hkv in ((4, 2), (16, 2)):        # 128 and 480 rows a KV head
        c = R.Cache(rng, dev, np.array(lens) + T, Hkv, 32, D, True)
        q, qh = R.rounded(rng, (2, Hq, T, D), True, dev)
        par = R.tree(rng, 2, T)
        desc = dreams.paged_desc(q, c.kd, c.vd, c.tabled, num_splits=8)
        n = dreams.paged_verify_attn_workspace_size(desc)
        assert n > 65536
        ws = torch.zeros(n, dtype=torch.uint8, device=dev)

        def call():
            return dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), R.ints(par, dev), num_splits=8,
                                            workspace=ws)
        ref = R.verify(qh, c.k, c.v, c.table, lens, par, R.ancestors(par), 0, 0, 1 / np.sqrt(D))
        for _ in range(2):
            R.check(*call(), ref, True, "workspace")
            dreams.workspace_status(ws)
            assert not ws[:65536].any()
        with pytest.raises(dreams.DreamsError) as e:
            dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), R.ints(par, dev), num_splits=8,
                                     workspace=ws[:n - 256])
        assert e.value.status == dreams.DREAMS_ERR_WORKSPACE
        try:
            dreams.set_wait_limit(0.0)
            call()
            torch.cuda.synchronize()
            with pytest.raises(dreams.DreamsError) as e:
                dreams.workspace_status(ws)
            assert e.value.status == dreams.DREAMS_ERR_DEVICE
        finally:
            dreams.set_wait_limit(0.2)
        ws[:65536].zero_()
        R.check(*call(), ref, True, "after a wait that gave up")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_upkeep_replayed(dev, dt):
    """Release, fork, reserve, append and commit in one graph: every replay does what the definition does."""
    rng = np.random.default_rng(14)
    B, width, P, ps, NL, Hkv, D, N = 5, 12, 70, 16, 2, 2, 64, 6
    t = R.Tables(B, width, P, ps)
    lens = np.array([70, 33, 0, 48, 100], np.int32)
    t.reserve(lens)
    t.kv_len[:] = lens
    on = t.on(dev)
    table, count, kv_len, ref = on
    k, v = random_bits(rng, (NL, P, Hkv, ps, D), dt, dev), random_bits(rng, (NL, P, Hkv, ps, D), dt, dev)
    new = [random_bits(rng, (NL, B, Hkv, N, D), dt, dev) for _ in range(2)]
    src, dst = R.ints([0, 1], dev), R.ints([2, 4], dev)
    path, alen = R.ints([[0, 2, 5, -1, -1, -1]] * B, dev), R.ints([2, 1, 0, 2, 2], dev)
    outs = dict(forked=torch.zeros(2, dtype=torch.int32, device=dev), room=torch.zeros(B, dtype=torch.int32, device=dev),
                after=torch.zeros(B, dtype=torch.int32, device=dev))

    def chain():
        dreams.pages_release(table, count, kv_len, ref, dst, ps)
        dreams.pages_fork(k, v, table, count, kv_len, ref, src, dst, granted=outs["forked"])
        dreams.pages_reserve(table, count, ref, kv_len + N, ps, granted=outs["room"])
        dreams.paged_append(new[0], new[1], k, v, table, kv_len)
        dreams.paged_kv_commit(k, v, table, kv_len, path, alen, kv_len_out=outs["after"])
        kv_len.copy_(outs["after"])

    start = [x.clone() for x in on + [k, v]]
    side = torch.cuda.Stream()               # every kernel once before the capture
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.synchronize()
    for x, y in zip(on + [k, v], start):
        x.copy_(y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain()
    pools = [bits(k).copy(), bits(v).copy()]
    for rep in range(4):
        g.replay()
        torch.cuda.synchronize()
        t.release([2, 4])
        granted, copies = t.fork([0, 1], [2, 4])
        assert outs["forked"].tolist() == granted == [1, 1]
        room = t.reserve(t.kv_len + N)
        assert outs["room"].tolist() == room == [1] * B, rep
        for w, x in zip(pools, new):
            xb = bits(x)
            for a, b, n in copies:
                w[:, b, :, :n] = w[:, a, :, :n]
            for b in range(B):
                for i in range(N):
                    j = int(t.kv_len[b]) + i
                    w[:, t.table[b, j // ps], :, j % ps] = xb[:, b, :, i]
                for n in range(int(alen[b]) + 1):
                    s, d = int(t.kv_len[b]) + [0, 2, 5][n], int(t.kv_len[b]) + n
                    w[:, t.table[b, d // ps], :, d % ps] = w[:, t.table[b, s // ps], :, s % ps]
        t.kv_len += alen.cpu().numpy() + 1
        assert outs["after"].tolist() == t.kv_len.tolist()
        t.same(on)
        assert np.array_equal(bits(k), pools[0]) and np.array_equal(bits(v), pools[1])


def test_empty_batches(dev):
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
    pages = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16, device=dev)
    q = torch.zeros((0, 4, 5, 64), dtype=torch.bfloat16, device=dev)
    out, lse = dreams.paged_verify_attn(q, pages, pages, z(0, 4), z(0), z(0, 5))
    assert out.shape == q.shape and lse.shape == (0, 4, 5)
    dreams.paged_prompt_attn(q, pages, pages, z(0, 4), z(0))
    dreams.paged_append(torch.zeros((0, 2, 5, 64), dtype=torch.bfloat16, device=dev),
                        torch.zeros((0, 2, 5, 64), dtype=torch.bfloat16, device=dev), pages, pages, z(0, 4), z(0))
    dreams.paged_append(torch.zeros((2, 2, 0, 64), dtype=torch.bfloat16, device=dev),
                        torch.zeros((2, 2, 0, 64), dtype=torch.bfloat16, device=dev), pages, pages, z(2, 4), z(2))
    assert dreams.paged_kv_commit(pages, pages, z(0, 4), z(0), z(0, 5), z(0)).shape == (0,)
    assert dreams.pages_reserve(z(0, 4), z(0), z(3), z(0), 16).shape == (0,)
    table, count, kv, ref = z(2, 4), z(2), z(2), z(3)
    assert dreams.pages_fork(pages, pages, table, count, kv, ref, z(0), z(0)).shape == (0,)
    dreams.pages_release(table, count, kv, ref, z(0), 16)
    torch.cuda.synchronize()


def test_refusals_on_the_device(dev):
    """What only device tensors reach: shapes, layouts, ranges."""
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
    pages = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16, device=dev)
    q = torch.zeros((2, 4, 5, 64), dtype=torch.bfloat16, device=dev)
    ok = dict(q=q, k_pages=pages, v_pages=pages, page_table=z(2, 4), kv_len=z(2))

    def bad(exception, match, **kw):
        for f, more in ((dreams.paged_verify_attn, dict(parent=z(2, 5))), (dreams.paged_prompt_attn, {})):
            with pytest.raises(exception, match=match):
                f(**{**ok, **more, **kw})
    bad(TypeError, "q must be", q=q.float())
    bad(ValueError, "contiguous", q=q.transpose(1, 2))
    bad(ValueError, "device tensor", q=q.cpu())
    bad(ValueError, "mismatch", page_table=z(3, 4))
    bad(ValueError, "kv_len must be", kv_len=z(3))
    bad(TypeError, "kv_len must be", kv_len=z(2).long())
    bad(ValueError, "differ in shape", v_pages=pages[:2])
    bad(ValueError, "dense", k_pages=torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16, device=dev)[..., :64],
        v_pages=torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16, device=dev)[..., :64])
    bad(ValueError, "layout", k_pages=torch.zeros((3, 2, 2, 16, 64), dtype=torch.bfloat16, device=dev)[:, 0])
    bad(ValueError, "window", window=2 ** 32)
    bad(ValueError, "window", sinks=-1)
    bad(dreams.DreamsError, "max_kv_len", max_kv_len=60)
    bad(dreams.DreamsError, "scale", scale=float("inf"))
    bad(ValueError, "lse must be", lse=torch.zeros((2, 4, 4), device=dev))
    with pytest.raises(ValueError, match="parent must be"):
        dreams.paged_verify_attn(**ok, parent=z(2, 4))
    with pytest.raises(dreams.DreamsError, match="parent or tree_mask"):
        dreams.paged_verify_attn(**ok)
    with pytest.raises(dreams.DreamsError, match="depths"):
        dreams.paged_verify_attn(**ok, window=4, tree_mask=torch.ones((2, 5, 1), dtype=torch.int64, device=dev))
    with pytest.raises(ValueError, match="row_len must be"):
        dreams.paged_prompt_attn(**ok, row_len=z(1))
    odd = torch.zeros((3, 2, 24, 64), dtype=torch.bfloat16, device=dev)
    bad(dreams.DreamsError, "page_size", k_pages=odd, v_pages=odd)
    new = torch.zeros((2, 2, 5, 64), dtype=torch.bfloat16, device=dev)
    for wrong in (new[:1], new[:, :1], new[..., :32], new.float(), new[None]):
        with pytest.raises((ValueError, TypeError)):
            dreams.paged_append(wrong, wrong, pages, pages, z(2, 4), z(2))
    with pytest.raises(ValueError, match="dense"):
        dreams.paged_append(new.transpose(2, 3).contiguous().transpose(2, 3), new.transpose(2, 3).contiguous().transpose(2, 3),
                            pages, pages, z(2, 4), z(2))
    with pytest.raises(dreams.DreamsError, match="strides"):
        wide = torch.zeros((2, 2, 5, 66), dtype=torch.bfloat16, device=dev)[..., :64]
        dreams.paged_append(wide, wide, pages, pages, z(2, 4), z(2))
    with pytest.raises(ValueError, match="refcount must be"):
        dreams.pages_fork(pages, pages, z(2, 4), z(2), z(2), z(4), z(1), z(1))
    with pytest.raises(ValueError, match="dst must be"):
        dreams.pages_fork(pages, pages, z(2, 4), z(2), z(2), z(3), z(1), z(2))
    with pytest.raises(ValueError, match="page_size"):
        dreams.pages_reserve(z(2, 4), z(2), z(3), z(2), 2 ** 32 + 16)
    with pytest.raises(dreams.DreamsError, match="page_size"):
        dreams.pages_reserve(z(2, 4), z(2), z(3), z(2), 48)
    kv = z(2)
    with pytest.raises(dreams.DreamsError, match="overlap"):
        dreams.paged_kv_commit(pages, pages, z(2, 4), kv, z(2, 5), z(2), kv_len_out=kv)


def test_workspaces_that_are_refused(dev):
    call = attention_case(np.random.default_rng(12), dev, torch.bfloat16, "verify")
    with pytest.raises(ValueError, match="workspace"):
        call(num_splits=3, workspace=torch.zeros(1 << 22, dtype=torch.uint8))
    with pytest.raises(ValueError, match="workspace"):
        call(num_splits=3, workspace=torch.zeros((1 << 22, 2), dtype=torch.uint8, device=dev)[:, 0])
    out, lse = call(num_splits=3)
    want = [bits(out), bits(lse)]
    # captured on a stream that is not the current one
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        outs = call(num_splits=3)
        with torch.cuda.stream(other):
            with pytest.raises(ValueError, match="workspace"):
                call(num_splits=3, stream=side, out=out, lse=lse)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip(outs, want):
            assert np.array_equal(bits(t), w)
        call(num_splits=3)


# heads, D, page, lengths, rows or nodes, window, sinks, mask
MANY_F32 = [
    ((16, 4), 64, 16, [50, 300, 0, 131], 70, 0, 0, False),
    ((16, 4), 128, 32, [50, 300, 0, 131], 70, 0, 0, True),               # masks that leave rows empty
    ((16, 4), 64, 16, [500, 33, 0, 131], 70, 40, 5, False),
    ((16, 2), 128, 64, [200, 33, 7, 600], 65, 3, 0, True),               # a window shorter than the tree is deep
    ((16, 16), 64, 16, [9 * i for i in range(29)], 9, 0, 0, False),      # 9 rows a KV head
    ((5, 5), 128, 16, [90] * 14, 60, 64, 33, False),
]


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("heads,D,ps,lens,N,window,sinks,masked", MANY_F32)
def test_many_rows_f32(dev, heads, D, ps, lens, N, window, sinks, masked, kind):
    """fp32 calls of more than 4096 rows (16 a compute unit), at least 8 of a KV head."""
    rng = np.random.default_rng(15)
    Hq, Hkv = heads
    B = len(lens)
    assert B * Hq * N >= 4096 and Hq // Hkv * N >= 8
    note(kind, heads, D, ps, lens, N, window, sinks, masked)
    q, qh = R.rounded(rng, (B, Hq, N, D), False, dev)
    if kind == "verify":
        c = R.Cache(rng, dev, np.array(lens) + N, Hkv, ps, D, False)
        par = R.tree(rng, B, N)
        see = R.ancestors(par)
        if masked:
            see &= rng.random(see.shape) < 0.5
            see[:, 0] = False
        out, lse = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), parent=R.ints(par, dev),
                                            tree_mask=torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None,
                                            window=window, sinks=sinks)
        torch.cuda.synchronize()
        ref = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
    else:
        rows = [int(x) for x in rng.integers(0, N + 1, size=B)]
        rows[0], rows[-1] = N, 0
        width = -(-(max(lens) + N) // ps)
        c = R.Cache(rng, dev, np.array(lens) + np.array(rows), Hkv, ps, D, False, width=width)
        for b in range(B):
            q[b, :, rows[b]:] = float("nan")
            qh[b, :, rows[b]:] = 0
        out, lse = dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), R.ints(rows, dev), window=window,
                                            sinks=sinks)
        torch.cuda.synchronize()
        ref = R.prompt(qh, c.k, c.v, c.table, lens, rows, window, sinks, 1 / np.sqrt(D))
    R.check(out, lse, ref, False, kind)
