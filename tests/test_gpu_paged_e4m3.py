"""A paged cache in 8 bits on the GPU: rows in, compacted, read back and forked, bit for bit against tests/e4m3_ref.py."""
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


def tables(B, lens, room, ps, spare=3):
    """Pages for every sequence's slots, in another order than their numbers."""
    need = [-(-(n + room) // ps) for n in lens]
    P = sum(need) + spare
    ids = np.random.default_rng(1).permutation(P)
    table = np.full((B, max(need)), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    return table, P


def fill(pool, table, lens, rng, dev, H, D):
    """The sequences' prefixes, appended on the host and put on the device as they are."""
    for b, n in enumerate(lens):
        for half in range(2):
            for layer in range(pool.codes.shape[1]):
                for g in range(H):
                    pool.append(half, layer, g, table[b], 0, rng.standard_normal((n, D)) if n else np.zeros((0, D)))
    for half, (c, s) in enumerate(((pool.k, pool.ks), (pool.v, pool.vs))):
        c.view(torch.uint8).copy_(torch.from_numpy(pool.codes[half]).to(dev))
        s.view(torch.uint8).copy_(torch.from_numpy(pool.scales[half]).to(dev))


def live_slots(pool, table, ends):
    live = np.zeros((pool.codes.shape[2], pool.ps), bool)
    for b, n in enumerate(ends):
        for j in range(n):
            live[table[b, j // pool.ps], j % pool.ps] = True
    return live


CASES = [
    # bf16 rows, NL, Hq, Hkv, D, R, interleaved, page, lengths, N, rows, tree, paired
    (True, 1, 0, 2, 64, 0, False, 16, [0, 15, 16, 40], 5, None, False, False),
    (True, 1, 4, 2, 128, 128, False, 16, [0, 1, 31, 40], 1, None, False, False),
    (True, 2, 0, 1, 128, 64, True, 32, [3, 0], 60, None, True, True),
    (False, 1, 3, 3, 64, 64, False, 64, [33, 7], 33, [33, 12], False, False),
    (True, 1, 7, 1, 128, 128, False, 16, [100, 7, 0], 70, [70, 0, 17], False, True),
    (False, 1, 0, 2, 80, 0, False, 16, [2, 20], 16, [3, 16], False, False),
    (True, 1, 2, 1, 256, 96, False, 16, [9], 21, None, True, False),
    (True, 1, 0, 1, 512, 512, True, 32, [17], 18, None, False, False),
    (False, 1, 2, 2, 16, 16, False, 256, [250, 3], 20, None, False, False),
]


@pytest.mark.parametrize("bf16,NL,Hq,H,D,rot,interleaved,ps,lens,N,rows,tree,paired", CASES)
def test_append(dev, bf16, NL, Hq, H, D, rot, interleaved, ps, lens, N, rows, tree, paired):
    rng = np.random.default_rng(2)
    note("append_e4m3", bf16, NL, Hq, H, D, rot, interleaved, ps, lens, N, rows, tree, paired)
    B = len(lens)
    live = [N] * B if rows is None else rows
    table, P = tables(B, lens, N, ps)
    pool = E.Pool8(rng, dev, NL, P, H, ps, D, paired)
    fill(pool, table, lens, rng, dev, H, D)
    kn, kh = E.spread_rows(rng, (NL, B, N, H, D), dev, bf16)
    vn, vh = E.spread_rows(rng, (NL, B, N, H, D), dev, bf16)
    kn, vn, vh = kn.transpose(2, 3), vn.transpose(2, 3), vh.swapaxes(2, 3)
    kv, rl = R.ints(lens, dev), None if rows is None else R.ints(rows, dev)
    kw = {}
    if rot:
        # (the rotation itself is tested by itself: here the same, in fp32)
        kw = dict(frequencies=dreams.rope_frequencies(rot, 1e4), interleaved=interleaved, amplitude=1.125,
                  parent=R.ints(R.tree(rng, B, N), dev) if tree else None)
        turn = lambda x: dreams.rope(x.float(), kv_len=kv, **kw)
        kh = np.stack([turn(kn[l]).double().cpu().numpy() for l in range(NL)])
    else:
        kh = kh.swapaxes(2, 3)
    q = E.spread_rows(rng, (B, N, Hq, D), dev, bf16)[0].transpose(1, 2) if Hq else None
    got = dreams.paged_append_e4m3(kn, vn, pool.k, pool.v, pool.ks, pool.vs, R.ints(table, dev), kv, row_len=rl, q=q, **kw)
    for half, x in enumerate((kh, vh)):
        for layer in range(NL):
            for b in range(B):
                for g in range(H):
                    pool.append(half, layer, g, table[b], lens[b], x[layer, b, g, :live[b]])
    pool.same(label="append")
    if q is not None:
        want = dreams.rope(q, kv_len=kv, **kw)
        for b in range(B):
            want[b, :, live[b]:] = 0
        assert torch.equal(got, want)
    # the same rows again find their scales: nothing changes
    dreams.paged_append_e4m3(kn, vn, pool.k, pool.v, pool.ks, pool.vs, R.ints(table, dev), kv, row_len=rl, **kw)
    pool.same(label="again")
    # read back, and past the end
    n = max(lens) + N + 3
    ends = np.array(lens) + live
    k, v = dreams.paged_read_e4m3(pool.k, pool.v, pool.ks, pool.vs, R.ints(table, dev), R.ints(ends, dev), n)
    assert k.dtype is torch.bfloat16 and k.shape == (NL, B, H, n, D) == v.shape
    for half, x in enumerate((k, v)):
        for layer in range(NL):
            for b in range(B):
                want = np.zeros((H, n, D))
                want[:, :ends[b]] = pool.slots(half, layer, table[b], ends[b])
                assert np.array_equal(x[layer, b].double().cpu().numpy(), want)


def test_blocks_at_the_ends_of_the_range(dev):
    """Blocks of zeros, of one nonzero value, at the border between two scales, with infinities and NaN, tiny and huge ones."""
    D, ps, H = 64, 16, 1
    border = [448.0, 448.0 * (1 + 2.0 ** -23), 449.0, 256.0, 512.0, 1.75, 1.7500001]
    blocks = [np.zeros((16, D))] + [np.full((16, D), x) for x in border]
    special = np.ones((16, D))
    special[3, 4], special[5, 6], special[7, 8], special[9, 9] = np.nan, np.inf, -np.inf, 1e-4
    only = np.full((16, D), np.nan)
    steps = np.zeros((16, D))
    steps[0] = np.resize(E.VALUES[:127], D)
    mids = (E.VALUES[:126] + E.VALUES[1:127]) / 2
    steps[1:3] = np.resize(mids, (2, D))            # ties
    steps[3:5] = np.resize(np.float32(mids) * np.float32(1 + 2.0 ** -22), (2, D))
    steps[5:7] = -np.resize(np.float32(mids) * np.float32(1 - 2.0 ** -22), (2, D))
    steps[8] = 448
    blocks += [special, only, steps, np.full((16, D), 3.4e38), np.full((16, D), 1e-38), np.full((16, D), 2.0 ** -149),
               np.full((16, D), 2.0 ** -126 * 1.9)]
    rows = np.concatenate(blocks)
    x = torch.from_numpy(rows).float().to(dev)
    rows = x.double().cpu().numpy()
    P = len(blocks)
    pool = E.Pool8(np.random.default_rng(3), dev, 1, P, H, ps, D)
    table = np.arange(P, dtype=np.int32)[None]
    new = x[None, None, None]
    dreams.paged_append_e4m3(new, -new, pool.k, pool.v, pool.ks, pool.vs, R.ints(table, dev), R.ints([0], dev))
    pool.append(0, 0, 0, table[0], 0, rows)
    pool.append(1, 0, 0, table[0], 0, -rows)
    pool.same(label="ends")
    for half in range(2):
        assert pool.scales[half, 0, :, 0, 0].min() >= 1 and pool.scales[half].max() <= 247


def test_rows_that_make_a_block_grow(dev):
    """One row after another into a block, each larger than the last: held rows move to the new scale."""
    rng = np.random.default_rng(4)
    D, ps, H, n = 64, 32, 2, 40
    pool = E.Pool8(rng, dev, 1, 3, H, ps, D)
    table = np.array([[2, 0]], np.int32)
    for j in range(n):
        size = 10.0 ** rng.uniform(-6, 6)
        kn = torch.from_numpy(size * rng.standard_normal((1, 1, H, 1, D))).to(torch.bfloat16).to(dev)
        vn = torch.from_numpy(size ** 3 * rng.standard_normal((1, 1, H, 1, D))).to(torch.bfloat16).to(dev)
        dreams.paged_append_e4m3(kn, vn, pool.k, pool.v, pool.ks, pool.vs, R.ints(table, dev), R.ints([j], dev))
        for half, x in enumerate((kn, vn)):
            for g in range(H):
                pool.append(half, 0, g, table[0], j, x[0, 0, g].double().cpu().numpy())
        pool.same(label=j)


def test_append_leaves_out_what_has_no_place(dev):
    rng = np.random.default_rng(5)
    B, H, N, D, ps, P = 4, 2, 20, 64, 16, 6
    table = np.array([[0, 1], [2, 99], [-1, 3], [4, 5]], np.int32)
    lens = [10, 8, 4, -3]
    pool = E.Pool8(rng, dev, 1, P, H, ps, D)
    kn, kh = E.spread_rows(rng, (1, B, H, N, D), dev, True)
    vn, vh = E.spread_rows(rng, (1, B, H, N, D), dev, True)
    dreams.paged_append_e4m3(kn, vn, pool.k, pool.v, pool.ks, pool.vs, R.ints(table, dev), R.ints(lens, dev))
    for half, x in enumerate((kh, vh)):
        for b in range(3):
            for g in range(H):
                pool.append(half, 0, g, table[b], lens[b], x[0, b, g])
    pool.same(label="no place")
    # reading them gives zeros
    k, v = dreams.paged_read_e4m3(pool.k[0], pool.v[0], pool.ks[0], pool.vs[0], R.ints(table, dev), R.ints([40, 40, 40, -1], dev), 40)
    for x in (k, v):
        assert (x[0, :, 32:] == 0).all() and (x[1, :, 16:] == 0).all() and (x[2, :, :16] == 0).all() and (x[3] == 0).all()


COMMITS = [
    # NL, H, D, page, lengths, T, paired
    (1, 2, 128, 16, [0, 15, 16, 40], 5, False),
    (2, 1, 64, 32, [3, 0, 77], 60, True),
    (1, 3, 64, 64, [33, 7], 128, False),
    (1, 1, 256, 16, [30, 5], 40, False),
    (1, 2, 16, 16, [21], 17, False),
    (1, 1, 80, 16, [4, 8], 33, False),
]


@pytest.mark.parametrize("NL,H,D,ps,lens,T,paired", COMMITS)
def test_commit(dev, NL, H, D, ps, lens, T, paired):
    rng = np.random.default_rng(6)
    note("commit_e4m3", NL, H, D, ps, lens, T, paired)
    B = len(lens)
    table, P = tables(B, lens, T, ps)
    pool = E.Pool8(rng, dev, NL, P, H, ps, D, paired)
    tab, kv = R.ints(table, dev), R.ints(lens, dev)
    for rep in range(3):
        kn, kh = E.spread_rows(rng, (NL, B, H, T, D), dev, True)
        vn, vh = E.spread_rows(rng, (NL, B, H, T, D), dev, True)
        if rep == 0:
            fill(pool, table, lens, rng, dev, H, D)
        par = R.tree(rng, B, T, depth=min(T - 1, 20), branch=3)
        path, taken = np.full((B, T), -1, np.int32), np.zeros(B, np.int32)
        dep = R.depths(par)
        for b in range(B):
            i = int(rng.integers(T))
            taken[b] = dep[b, i]
            while i >= 0:
                path[b, dep[b, i]] = i
                i = int(par[b, i])
        if rep == 1 and T > 8:      # entries that are skipped, lengths out of range
            path[0, :6] = [0, 3, 1, 2 ** 30, -5, 7]
            taken[0], taken[-1] = 5, 10 ** 6
        dreams.paged_append_e4m3(kn, vn, pool.k, pool.v, pool.ks, pool.vs, tab, kv)
        out = dreams.paged_kv_commit_e4m3(pool.k, pool.v, pool.ks, pool.vs, tab, kv, R.ints(path, dev), R.ints(taken, dev))
        A = np.clip(taken, 0, T - 1)
        assert out.tolist() == (np.array(lens) + A + 1).tolist()
        for half, x in enumerate((kh, vh)):
            for layer in range(NL):
                for b in range(B):
                    for g in range(H):
                        pool.append(half, layer, g, table[b], lens[b], x[layer, b, g])
                        pool.commit(half, layer, g, table[b], lens[b], path[b], int(A[b]))
        pool.same(live_slots(pool, table, np.array(lens) + A + 1), "commit %d" % rep)
        pool.codes[0], pool.codes[1] = (x.view(torch.uint8).cpu().numpy() for x in (pool.k, pool.v))
        pool.scales[0], pool.scales[1] = (x.view(torch.uint8).cpu().numpy() for x in (pool.ks, pool.vs))


@pytest.mark.parametrize("NL,H,ps,D,paired", [(1, 2, 16, 64, False), (3, 1, 64, 128, True), (2, 4, 256, 64, False)])
def test_fork(dev, NL, H, ps, D, paired):
    rng = np.random.default_rng(7)
    B, P = 6, 40
    t = R.Tables(B, 6, P, ps)
    lens = [ps * 2 + 5, ps, 0, ps + ps - 1, 0, 0]
    t.reserve(lens)
    t.kv_len[:] = lens
    pool = E.Pool8(rng, dev, NL, P, H, ps, D, paired)
    on = t.on(dev)
    granted, copies = t.fork([0, 1, 3], [4, 5, 2])
    got = dreams.pages_fork_e4m3(pool.k, pool.v, pool.ks, pool.vs, *on, R.ints([0, 1, 3], dev), R.ints([4, 5, 2], dev))
    assert got.tolist() == granted == [1, 1, 1]
    for a, b, n in copies:
        pool.codes[:, :, b, :, :n] = pool.codes[:, :, a, :, :n]
        pool.scales[:, :, b, :, :-(-n // 16)] = pool.scales[:, :, a, :, :-(-n // 16)]
    t.same(on)
    pool.same(label="fork")


def test_replayed_and_on_another_stream(dev):
    """A step captured and replayed with other rows, lengths and paths, and the same calls on a stream of their own."""
    rng = np.random.default_rng(8)
    B, Hq, H, T, D, ps = 2, 4, 2, 9, 128, 16
    table = np.array([[0, 1, 2, 3], [4, 5, 6, 7]], np.int32)
    tab, kv = R.ints(table, dev), R.ints([20, 3], dev)
    kn, vn = (E.spread_rows(rng, (B, H, T, D), dev, True)[0] for _ in range(2))
    q, freq = R.rounded(rng, (B, Hq, T, D), True, dev)[0], dreams.rope_frequencies(D)
    par = R.ints(R.tree(rng, B, T), dev)
    path, taken = R.ints([[0, 2, 5, -1, -1, -1, -1, -1, -1], [0, 1, 3, 8, -1, -1, -1, -1, -1]], dev), R.ints([2, 3], dev)
    start = E.Pool8(rng, dev, 1, 8, H, ps, D)
    pool = [x[0].clone() for x in (start.k, start.v, start.ks, start.vs)]

    def reset():
        for x, y in zip(pool, (start.k, start.v, start.ks, start.vs)):
            x.view(torch.uint8).copy_(y[0].view(torch.uint8))

    def run(**kw):
        turned = dreams.paged_append_e4m3(kn, vn, *pool, tab, kv, frequencies=freq, q=q, parent=par, **kw)
        held = dreams.paged_kv_commit_e4m3(*pool, tab, kv, path, taken, **kw)
        return [turned, held, *dreams.paged_read_e4m3(*pool, tab, held, 40, **kw)]

    same = lambda a, b: all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
                            for x, y in zip(a, b))
    reset()
    want = run()
    reset()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(stream=side)
    side.synchronize()
    assert same(got, want)
    reset()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for rep in range(3):
        kn.normal_(), q.normal_()
        kv.copy_(torch.tensor([20 + rep, 3 + 7 * rep], dtype=torch.int32))
        taken.copy_(torch.tensor([rep, 3 - rep], dtype=torch.int32))
        reset()
        want, wpool = run(), None
        wpool = [x.clone() for x in pool]
        reset()
        g.replay()
        torch.cuda.synchronize()
        assert same(out, want) and same(pool, wpool)


def test_refusals_on_the_device(dev):
    pool = E.Pool8(np.random.default_rng(1), dev, 1, 4, 2, 32, 64)
    k, v, ks, vs = (x[0] for x in (pool.k, pool.v, pool.ks, pool.vs))
    tab, kv = R.ints([[0], [1]], dev), R.ints([0, 0], dev)
    x = torch.zeros((2, 2, 4, 64), dtype=torch.bfloat16, device=dev)
    freq = dreams.rope_frequencies(64)
    ok = dict(k_new=x, v_new=x, k_pages=k, v_pages=v, k_scales=ks, v_scales=vs, page_table=tab, kv_len=kv)
    for bad, error in ((dict(k_pages=k.view(torch.uint8), v_pages=v.view(torch.uint8)), TypeError),
                       (dict(k_pages=x), TypeError), (dict(k_scales=ks.view(torch.uint8)), TypeError),
                       (dict(k_scales=ks[:3]), ValueError), (dict(k_scales=ks.cpu()), ValueError),
                       (dict(k_scales=ks[:, :, :1], v_scales=vs[:, :, :1]), ValueError),
                       (dict(k_scales=ks[:1].expand(4, 2, 2), v_scales=vs[:1].expand(4, 2, 2)), ValueError),
                       (dict(k_scales=ks.transpose(1, 2).contiguous().transpose(1, 2)), ValueError),
                       (dict(k_new=x.half(), v_new=x.half()), TypeError), (dict(v_new=x.float()), TypeError),
                       (dict(q=x), ValueError), (dict(parent=kv), ValueError), (dict(k_new=None), TypeError),
                       (dict(q=x.float(), frequencies=freq), TypeError), (dict(kv_len=kv[:1]), ValueError),
                       (dict(frequencies=dreams.rope_frequencies(128)), dreams.DreamsError)):
        with pytest.raises(error):
            dreams.paged_append_e4m3(**{**ok, **bad})
    dense = torch.zeros((4, 2, 32, 64), dtype=torch.bfloat16, device=dev)
    for call in (lambda: dreams.paged_append(x, x, k, v, tab, kv),
                 lambda: dreams.paged_prompt_attn(x, k, v, tab, kv), lambda: dreams.paged_kv_commit(k, v, tab, kv, tab, kv),
                 lambda: dreams.paged_read_e4m3(dense, dense, ks, vs, tab, kv, 5),
                 lambda: dreams.pages_fork(k, v, tab, kv, kv, R.ints([0] * 4, dev), kv, kv)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        dreams.paged_read_e4m3(k, v, ks, vs, tab, kv, -1)
    empty = dreams.paged_read_e4m3(k, v, ks, vs, tab[:0], kv[:0], 5)
    assert empty[0].shape == (0, 2, 5, 64)
    assert dreams.paged_read_e4m3(k, v, ks, vs, tab, kv, 0)[1].shape == (2, 2, 0, 64)
