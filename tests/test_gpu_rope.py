"""Rotary positions on the GPU: by themselves, and on the way into a paged cache, against tests/e4m3_ref.py."""
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


def laid_out(x, order, dev, dt):
    """x [B,H,N,D] as a tensor of that shape in memory order `order` of its axes, rows dense."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dt).to(dev)
    return t.permute(order).contiguous().permute([order.index(i) for i in range(4)])


# B, H, N, D, R, interleaved, memory order, gain
SHAPES = [
    (1, 1, 1, 64, 64, False, (0, 1, 2, 3), 1.0),
    (4, 32, 1, 128, 128, False, (0, 2, 1, 3), 1.0),
    (2, 3, 17, 128, 128, True, (0, 2, 1, 3), 1.25),
    (3, 5, 33, 64, 32, False, (0, 1, 2, 3), 0.5),
    (2, 7, 9, 80, 80, False, (2, 1, 0, 3), 1.0),
    (2, 2, 40, 96, 48, True, (0, 2, 1, 3), 1.0),
    (1, 2, 5, 72, 16, False, (0, 2, 1, 3), -1.0),
    (2, 1, 130, 128, 64, True, (1, 2, 0, 3), 1.1),
    (1, 40, 257, 128, 128, False, (0, 2, 1, 3), 1.0),
    (5, 28, 64, 128, 112, False, (0, 2, 1, 3), 1.0),
]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,H,N,D,rot,interleaved,order,gain", SHAPES)
def test_rope(dev, B, H, N, D, rot, interleaved, order, gain, dt):
    rng = np.random.default_rng(3)
    note("rope", B, H, N, D, rot, interleaved, order, dt)
    x = laid_out(rng.standard_normal((B, H, N, D)), order, dev, dt)
    xh, bf16 = x.double().cpu().numpy(), dt is torch.bfloat16
    freq = dreams.rope_frequencies(rot, 5e5)
    fh = freq.cpu().numpy()
    base = rng.integers(0, 40000, size=B)
    given = rng.integers(-2 ** 31, 2 ** 31, size=(B, N))
    tree = R.tree(rng, B, min(N, 128))
    kv = R.ints(base, dev)

    def check(got, where, label):
        want, size, far = E.rotate(xh, where[:, None], fh, gain, interleaved)
        E.check_rotation(got.double().cpu().numpy(), want, size, far, bf16, label)

    kw = dict(interleaved=interleaved, amplitude=gain)
    out = dreams.rope(x, freq, kv_len=kv, **kw)
    assert out.is_contiguous()
    check(out, base[:, None] + np.arange(N), "in order")
    assert torch.equal(x.double().cpu(), torch.from_numpy(xh))
    check(dreams.rope(x, freq, positions=R.ints(given, dev), **kw), given, "given")
    if N <= 128:
        check(dreams.rope(x, freq, kv_len=kv, parent=R.ints(tree, dev), **kw), base[:, None] + R.depths(tree), "tree")
    # into a view of another layout with rows around it, and in place
    wide = torch.full((B, N + 2, H + 1, D), 7.0, dtype=dt, device=dev)
    to = wide[:, 1:N + 1, :H].transpose(1, 2)
    assert dreams.rope(x, freq, kv_len=kv, out=to, **kw) is to
    assert torch.equal(to, out)
    wide[:, 1:N + 1, :H] = 7.0
    assert (wide == 7.0).all()
    assert dreams.rope(x, freq, kv_len=kv, out=x, **kw) is x and torch.equal(x, out)


def test_other_columns_and_special_values(dev):
    """Columns past rotary_dim keep their bits; position 0 leaves a row as it is (but for the gain); a NaN or an infinity
    stays within its pair."""
    rng = np.random.default_rng(5)
    x, _ = R.rounded(rng, (1, 2, 6, 64), True, dev)
    x[..., 32:] = torch.from_numpy(rng.integers(-2 ** 15, 2 ** 15, size=(1, 2, 6, 32)).astype(np.int16)).to(dev).view(
        torch.bfloat16)
    x[0, 0, 3, 5], x[0, 1, 4, 20] = float("nan"), float("inf")
    freq = dreams.rope_frequencies(32)
    out = dreams.rope(x, freq, positions=R.ints([[0, 1, 2, 3, 4, 5]], dev))
    assert torch.equal(out[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16))
    assert torch.equal(out[:, :, 0, :32], x[:, :, 0, :32])
    bad = ~torch.isfinite(out[..., :32])
    want = torch.zeros_like(bad)
    want[0, 0, 3, [5, 21]] = want[0, 1, 4, [4, 20]] = True
    assert torch.equal(bad, want)


def test_a_position_turned_back(dev):
    """Rotations add up: p and then -p gives the row again, to the rotations' roundings."""
    rng = np.random.default_rng(6)
    x, xh = R.rounded(rng, (2, 3, 50, 128), False, dev)
    freq = dreams.rope_frequencies(128, 1e4, "parts", 8.0, 4096)
    p = rng.integers(0, 100000, size=(2, 50))
    there = dreams.rope(x, freq, positions=R.ints(p, dev))
    back = dreams.rope(there, freq, positions=R.ints(-p, dev)).double().cpu().numpy()
    _, size, far = E.rotate(xh, p[:, None], freq.cpu().numpy(), 1.0, False)
    # twice the tolerance of one rotation, of pairs up to sqrt(2) as large
    assert (np.abs(back - xh) <= 2 * 1.5 * size * (8 * 2.0 ** -24 + 2 * np.pi * 2.0 ** -51 * far)).all()


APPENDS = [
    # dt, NL, Hq, Hkv, D, R, interleaved, page, lengths, N, rows, tree, paired
    (torch.bfloat16, 1, 4, 2, 128, 128, False, 16, [0, 15, 16, 40], 5, None, False, False),
    (torch.bfloat16, 1, 8, 8, 64, 32, True, 32, [3, 0], 60, None, True, True),
    (torch.bfloat16, 1, 7, 1, 128, 128, False, 16, [100, 7, 0], 130, [130, 0, 17], False, False),
    (torch.float32, 1, 4, 4, 64, 64, True, 64, [60, 1], 9, [9, 3], True, False),
    (torch.float32, 1, 2, 1, 80, 80, False, 16, [2], 1, None, False, True),
    (torch.bfloat16, 3, 0, 2, 128, 64, False, 16, [9, 30], 12, [12, 5], False, False),
    (torch.bfloat16, 1, 32, 8, 128, 128, False, 16, [1000, 31, 0, 5], 1, None, False, False),
]


@pytest.mark.parametrize("dt,NL,Hq,Hkv,D,rot,interleaved,ps,lens,N,rows,tree,paired", APPENDS)
def test_append_rope(dev, dt, NL, Hq, Hkv, D, rot, interleaved, ps, lens, N, rows, tree, paired):
    """Bit for bit what the rotation alone and the append alone do."""
    rng = np.random.default_rng(8)
    note("append_rope", dt, NL, Hq, Hkv, D, rot, interleaved, ps, lens, N, rows, tree, paired)
    B = len(lens)
    live = [N] * B if rows is None else rows
    table = R.Tables(B, -(-(max(lens) + N) // ps) + 1, 60 + sum(lens) // ps, ps)
    table.reserve(np.array(lens) + N)
    tab, P = R.ints(table.table, dev), len(table.ref)
    new = lambda: torch.from_numpy(rng.standard_normal((NL, B, N, Hkv, D))).to(dt).to(dev).transpose(2, 3)
    kn, vn = new(), new()
    shape = (NL, P, 2, Hkv, ps, D) if paired else (2, NL, P, Hkv, ps, D)
    pool = torch.from_numpy(rng.standard_normal(shape)).to(dt).to(dev)
    other = pool.clone()
    halves = lambda t: (t[:, :, 0], t[:, :, 1]) if paired else (t[0], t[1])
    (k, v), (k2, v2) = halves(pool), halves(other)
    kv, rl = R.ints(lens, dev), None if rows is None else R.ints(rows, dev)
    par = R.ints(R.tree(rng, B, N), dev) if tree else None
    freq = dreams.rope_frequencies(rot, 1e6)
    kw = dict(parent=par, interleaved=interleaved, amplitude=1.0625)
    q = torch.from_numpy(rng.standard_normal((B, N, Hq, D))).to(dt).to(dev).transpose(1, 2) if Hq else None
    got = dreams.paged_append_rope(kn, vn, k, v, tab, kv, freq, row_len=rl, q=q, **kw)
    turned = torch.stack([dreams.rope(kn[l], freq, kv_len=kv, **kw) for l in range(NL)])
    dreams.paged_append(turned, vn.contiguous(), k2, v2, tab, kv, row_len=rl)
    assert torch.equal(pool, other)
    assert (got is None) == (q is None)
    if q is not None:
        want = dreams.rope(q, freq, kv_len=kv, **kw)
        for b in range(B):
            want[b, :, live[b]:] = 0
        assert torch.equal(got, want) and got.is_contiguous()
    if NL == 1:     # one layer's pages, without NL; the same again changes nothing
        assert dreams.paged_append_rope(kn[0], vn[0], k[0], v[0], tab, kv, freq, row_len=rl, **kw) is None
        assert torch.equal(pool, other)


def test_append_rope_leaves_out_what_has_no_place(dev):
    """Rows past the table, on pages outside the pool, of a negative length: not written; their queries are rotated."""
    rng = np.random.default_rng(9)
    B, H, N, D, ps, P = 4, 2, 20, 64, 16, 6
    tab = R.ints([[0, 1], [2, 99], [-1, 3], [4, 5]], dev)
    lens = [10, 8, 4, -3]
    kn, vn, q = (torch.from_numpy(rng.standard_normal((B, H, N, D))).float().to(dev) for _ in range(3))
    k = torch.full((P, H, ps, D), 7.0, device=dev)
    v = k.clone()
    freq = dreams.rope_frequencies(D)
    got = dreams.paged_append_rope(kn, vn, k, v, tab, R.ints(lens, dev), freq, q=q)
    assert torch.equal(got, dreams.rope(q, freq, kv_len=R.ints(lens, dev)))
    turned = dreams.rope(kn, freq, kv_len=R.ints(lens, dev))
    want_k, want_v = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    for b, pages in enumerate(([0, 1], [2, None], [None, 3])):
        for i in range(N):
            slot = lens[b] + i
            if slot // ps < 2 and pages[slot // ps] is not None:
                want_k[pages[slot // ps], :, slot % ps] = turned[b, :, i]
                want_v[pages[slot // ps], :, slot % ps] = vn[b, :, i]
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


@pytest.mark.parametrize("captured", [False, True])
def test_on_another_stream_and_replayed(dev, captured):
    rng = np.random.default_rng(10)
    B, Hq, H, N, D, ps = 2, 4, 2, 7, 128, 16
    tab, kv = R.ints([[0, 1, 2], [3, 4, 5]], dev), R.ints([20, 3], dev)
    kn, vn = (R.rounded(rng, (B, H, N, D), True, dev)[0] for _ in range(2))
    q, freq = R.rounded(rng, (B, Hq, N, D), True, dev)[0], dreams.rope_frequencies(D)
    k = torch.zeros((6, H, ps, D), dtype=torch.bfloat16, device=dev)
    v = torch.zeros_like(k)
    run = lambda **kw: (dreams.rope(q, freq, kv_len=kv, **kw),
                        dreams.paged_append_rope(kn, vn, k, v, tab, kv, freq, q=q, **kw))
    want = run()
    wk, wv = k.clone(), v.clone()
    torch.cuda.synchronize()
    if not captured:
        side = torch.cuda.Stream()
        k.zero_(), v.zero_()
        torch.cuda.synchronize()
        got = run(stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(k, wk) and torch.equal(v, wv)
        return
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for rep in range(3):
        q.normal_(), kn.normal_()
        kv.copy_(torch.tensor([20 + rep, 3 + 5 * rep], dtype=torch.int32))
        k.zero_(), v.zero_()
        g.replay()
        torch.cuda.synchronize()
        gk, gv = k.clone(), v.clone()
        k.zero_(), v.zero_()
        want = run()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(gk, k) and torch.equal(gv, v)


def test_refusals_on_the_device(dev):
    x = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16, device=dev)
    freq, kv = dreams.rope_frequencies(64), R.ints([0, 0], dev)
    for bad, error in ((dict(frequencies=freq.float()), TypeError), (dict(frequencies=freq.cpu()), ValueError),
                       (dict(kv_len=None), dreams.DreamsError), (dict(kv_len=R.ints([0], dev)), ValueError),
                       (dict(positions=R.ints([[0] * 4], dev)), ValueError), (dict(x=x[:, :, :, ::2]), ValueError),
                       (dict(x=x.half()), TypeError), (dict(x=x[0]), ValueError), (dict(x=x.cpu()), ValueError),
                       (dict(frequencies=dreams.rope_frequencies(128)), dreams.DreamsError),
                       (dict(frequencies=dreams.rope_frequencies(24)), dreams.DreamsError),
                       (dict(amplitude=float("nan")), dreams.DreamsError), (dict(out=x.float()), ValueError),
                       (dict(out=x[:1].expand(2, 3, 4, 64)), dreams.DreamsError),
                       (dict(x=x.view(2, 3, 2, 128)[..., :68]), dreams.DreamsError)):
        args = dict(x=x, frequencies=freq, kv_len=kv)
        args.update(bad)
        with pytest.raises(error):
            dreams.rope(args.pop("x"), args.pop("frequencies"), **args)
    long = torch.zeros((1, 1, 129, 64), dtype=torch.bfloat16, device=dev)
    with pytest.raises(dreams.DreamsError, match="tree nodes"):
        dreams.rope(long, freq, kv_len=kv[:1], parent=R.ints([[-1] + [0] * 128], dev))
    pages = torch.zeros((4, 3, 16, 64), dtype=torch.bfloat16, device=dev)
    tab = R.ints([[0], [1]], dev)
    call = lambda **kw: dreams.paged_append_rope(x, x, pages, pages, tab, kv, freq, **kw)
    for kw, error in ((dict(q=x.float()), TypeError), (dict(q=x[:1]), ValueError), (dict(q=x[:, :, :3]), ValueError),
                      (dict(q_out=x), ValueError), (dict(q=x, q_out=x.float()), TypeError),
                      (dict(q=x, q_out=x[:, :2]), ValueError)):
        with pytest.raises(error):
            call(**kw)
    layers = pages[None].repeat(2, 1, 1, 1, 1)
    with pytest.raises(dreams.DreamsError, match="one layer"):
        dreams.paged_append_rope(x[None].repeat(2, 1, 1, 1, 1), x[None].repeat(2, 1, 1, 1, 1), layers, layers, tab, kv, freq, q=x)
    assert dreams.rope(x[:0], freq, kv_len=kv[:0]).shape == (0, 3, 4, 64)
    assert dreams.rope(x[:, :, :0], freq, kv_len=kv).shape == (2, 3, 0, 64)
