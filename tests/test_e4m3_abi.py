"""Refusals of the rotary and 8-bit entry points on the CPU, the frequencies' formulas, and pins of the 8-bit definitions
that the GPU tests compare with.  No kernel runs here."""
import ctypes

import numpy as np
import pytest
import torch

import e4m3_ref as E
from test_paged_abi import D, FAKE, ODD, POOLS, pool  # noqa: F401  (D: the fixture)

FAR = ctypes.c_void_p(0x200000)


def rope(D, **kw):
    d = dict(rotary_dim=64, interleaved=0, frequencies=0x100000, positions=None, parent=None, amplitude=1.0)
    d.update(kw)
    return D.Rope(**d)


ROPES = [(dict(rotary_dim=0), -1), (dict(rotary_dim=-16), -1), (dict(rotary_dim=144), -1), (dict(rotary_dim=24), -2),
         (dict(interleaved=2), -1), (dict(amplitude=float("inf")), -1), (dict(amplitude=float("nan")), -1),
         (dict(frequencies=None), -1), (dict(frequencies=0x100004), -1), (dict(positions=0x100002), -1),
         (dict(parent=0x100002), -1)]


def test_rope(D):
    lib = D.lib()

    def call(r, B=2, H=4, N=5, dim=128, dt=1, x=FAKE, xs=(4096, 1024, 128), kv=FAKE, out=FAR, os=(4096, 1024, 128)):
        three = ctypes.c_int64 * 3
        return lib.dreams_rope(None if r is None else ctypes.byref(r), B, H, N, dim, dt, x, None if xs is None else three(*xs),
                               kv, out, None if os is None else three(*os), None)

    for kw, status in ROPES:
        assert call(rope(D, **kw)) == status, kw
        assert lib.dreams_last_error_message().decode() != ""
    assert call(None) == -1
    for kw, status in ((dict(B=-1), -1), (dict(H=0), -1), (dict(N=-1), -1), (dict(dim=0), -1), (dict(dim=516), -2),
                       (dict(dim=68), -2), (dict(dim=520), -2), (dict(dt=2), -1), (dict(dt=7), -1), (dict(xs=None), -1),
                       (dict(os=None), -1), (dict(xs=(4096, 1024, 129)), -1), (dict(os=(4096, -1024, 128)), -1),
                       (dict(os=(4096, 0, 128)), -1), (dict(x=None), -1), (dict(out=None), -1), (dict(x=ODD), -1),
                       (dict(out=ODD), -1), (dict(kv=None), -1), (dict(kv=ODD), -1), (dict(B=70000), -2),
                       (dict(N=1 << 29), -2), (dict(out=FAKE, os=(4096, 128, 512)), -1)):
        assert call(rope(D), **kw) == status, kw
    assert call(rope(D, parent=0x100000), N=129) == -1 and b"tree nodes" in lib.dreams_last_error_message()
    assert call(rope(D), B=0) == 0 and call(rope(D), N=0) == 0
    assert call(rope(D), dt=0, dim=68) == -2 and call(rope(D), dt=0, dim=520) == -2
    at = lambda x: ctypes.c_void_p(0x100000 + x)
    dense = (4 * 5 * 128, 5 * 128, 128)
    for kw in (dict(out=at(256)), dict(out=at(-256)), dict(xs=dense, out=at(2 * 4 * 5 * 128 * 2 - 16), os=dense),
               dict(xs=(0, 0, 0), out=at(-256), os=dense), dict(xs=(4096, 512, 2048), os=dense, out=at(1024))):
        kw = dict(dict(xs=dense, os=dense), **kw)
        assert call(rope(D), **kw) == -1 and b"overlap" in lib.dreams_last_error_message(), kw
    # (fp32 rows have twice the units: more than 2^31 of them, fewer in bf16 -- which the null pointer then refuses)
    assert call(rope(D), N=1 << 25, dt=0, x=None, B=1) == -2 and call(rope(D), N=1 << 25, x=None, B=1) == -1


def test_frequencies(D):
    got = D.rope_frequencies(128, 5e5, device="cpu").numpy()
    plain = 5e5 ** (-2 * np.arange(64) / 128)
    assert np.allclose(got, plain, rtol=2e-15, atol=0)
    assert np.allclose(D.rope_frequencies(128, 5e5, "linear", 4.0, device="cpu").numpy(), plain / 4, rtol=2e-15, atol=0)
    turns = 4096 * plain / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    parts = D.rope_frequencies(128, 5e5, "parts", 8.0, 4096, device="cpu").numpy()
    assert np.allclose(parts, plain * (keep + (1 - keep) / 8), rtol=1e-14, atol=0)
    assert (parts[turns >= 32] == got[turns >= 32]).all() and np.allclose(parts[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    for kw in (dict(rotary_dim=1), dict(rotary_dim=0), dict(scaling="other")):
        with pytest.raises(ValueError):
            D.rope_frequencies(**{"rotary_dim": 64, "device": "cpu", **kw})
    for kw in (dict(rotary_dim=63), dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.0),
               dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, trained_len=4096, low=5.0, high=5.0),
               dict(scaling="parts", factor=2.0, trained_len=4096, low=float("nan")),
               dict(scaling="parts", factor=2.0, trained_len=float("inf"))):
        with pytest.raises(D.DreamsError):
            D.rope_frequencies(**{"rotary_dim": 64, "device": "cpu", **kw})
    f = D.lib().dreams_rope_frequencies
    assert f(64, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == -1 and f(64, 1e4, 3, 1.0, 0.0, 0.0, 0.0, FAKE) == -1


def test_appends(D):
    lib = D.lib()
    st4 = lambda s: None if s is None else (ctypes.c_int64 * 4)(*s)

    def queries(**kw):
        d = dict(q=0x100000, out=0x300000, num_q_heads=8, strides=(ctypes.c_int64 * 3)(8192, 128, 1024))
        d.update(kw)
        return D.RopeQueries(**d)

    def plain(p, r=None, q=None, k=FAKE, v=FAKE, n=5, strides=(4096, 1024, 512, 128), table=FAKE, kv=FAKE, rows=None, kp=FAKE,
              vp=FAKE):
        r = rope(D) if r is None else r
        return lib.dreams_paged_append_rope(ctypes.byref(p), ctypes.byref(r), None if q is None else ctypes.byref(q), k, v, n,
                                            st4(strides), table, kv, rows, kp, vp, None)

    def eight(p, r=None, q=None, k=FAKE, v=FAKE, n=5, strides=(4096, 1024, 512, 128), table=FAKE, kv=FAKE, rows=None, kp=FAKE,
              vp=FAKE, s=None, dt=1):
        s = D.PageScales(0x100000, 0x100000, 0, 0) if s is None else s
        p.dtype = D.DREAMS_E4M3 if p.dtype == D.DREAMS_BF16 else p.dtype
        return lib.dreams_paged_append_e4m3(ctypes.byref(p), ctypes.byref(s), None if r is None else ctypes.byref(r),
                                            None if q is None else ctypes.byref(q), dt, k, v, n, st4(strides), table, kv, rows,
                                            kp, vp, None)

    wide = [x for x in POOLS if x[0] not in (dict(head_dim=512), dict(page_stride=4100))]
    for f, one in ((plain, dict()), (eight, dict())):
        for kw, status in wide:
            assert f(pool(D, **kw)) == status, (f.__name__, kw)
        assert f(pool(D, batch=0)) == 0 and f(pool(D), n=0) == 0 and f(pool(D), n=-1) == -1
        for kw, status in ROPES:
            assert f(pool(D), r=rope(D, **kw)) == status, (f.__name__, kw)
        for bad in (None, (-8, 1024, 512, 128), (4096, 1028, 512, 128), (4096, 1024, 512, 129), (4096, 1024, 1 << 50, 128)):
            assert f(pool(D), strides=bad) == -1
        for name in ("k", "v", "table", "kv", "kp", "vp"):
            assert f(pool(D), **{name: None}) == -1 and f(pool(D), **{name: ODD}) == -1
        assert f(pool(D), rows=ODD) == -1 and f(pool(D), n=1 << 28) == -2
        assert f(pool(D), r=rope(D), q=queries()) == -1 and b"one layer" in lib.dreams_last_error_message()
        for kw in (dict(num_q_heads=0), dict(q=None), dict(out=None), dict(q=0x100002), dict(out=0x100008),
                   dict(strides=(ctypes.c_int64 * 3)(8192, 129, 1024)), dict(strides=(ctypes.c_int64 * 3)(8192, 128, -1024))):
            assert f(pool(D, num_layers=1), r=rope(D), q=queries(**kw)) == -1, kw
        for kw in (dict(out=0x100000), dict(out=0x100000 + 2 * 8192), dict(q=0x300000 + 2 * 2 * 8 * 5 * 128 - 16)):
            assert f(pool(D, num_layers=1), r=rope(D), q=queries(**kw)) == -1, kw
            assert b"overlap" in lib.dreams_last_error_message()
    assert plain(pool(D, dtype=D.DREAMS_E4M3)) == -1
    assert lib.dreams_paged_append_rope(ctypes.byref(pool(D)), None, None, FAKE, FAKE, 5, st4((4096, 1024, 512, 128)), FAKE, FAKE,
                                        None, FAKE, FAKE, None) == -1
    assert eight(pool(D, num_layers=1), q=queries()) == -1 and b"need rope" in lib.dreams_last_error_message()
    assert eight(pool(D, dtype=D.DREAMS_F32)) == -1 and eight(pool(D), dt=2) == -1
    assert eight(pool(D, head_dim=520)) == -2 and eight(pool(D, head_dim=72)) == -2
    # (a wave a block of 16 rows of a head: 2^32 threads and more, however short the rows)
    assert eight(pool(D, head_dim=16), n=1 << 27) == -2 and eight(pool(D, head_dim=16), n=1 << 25, k=None) == -1
    for s in (D.PageScales(None, 0x100000, 0, 0), D.PageScales(0x100000, None, 0, 0), D.PageScales(0x100000, 0x100000, 0, 1),
              D.PageScales(0x100000, 0x100000, 0, -4), D.PageScales(0x100000, 0x100000, 100, 0),
              D.PageScales(0x100000, 0x100000, 0, 1 << 60), D.PageScales(0x100000, 0x100000, -1, 0)):
        assert eight(pool(D), s=s) == -1


def test_commits_reads_and_forks(D):
    lib = D.lib()
    good = lambda: D.PageScales(0x100000, 0x100000, 0, 0)

    def commit(p, s=None, kp=FAKE, vp=FAKE, table=FAKE, kv=FAKE, path=FAKE, alen=FAKE, ps=60, out=FAR):
        return lib.dreams_paged_kv_commit_e4m3(ctypes.byref(p), ctypes.byref(s or good()), kp, vp, table, kv, path, alen, ps,
                                               out, None)

    def read(p, s=None, kp=FAKE, vp=FAKE, table=FAKE, kv=FAKE, n=9, ko=FAR, vo=FAR):
        return lib.dreams_paged_read_e4m3(ctypes.byref(p), ctypes.byref(s or good()), kp, vp, table, kv, n, ko, vo, None)

    def fork(p, s=None, kp=FAKE, vp=FAKE, table=FAKE, count=FAKE, kv=FAKE, ref=FAKE, n=2, src=FAKE, dst=FAKE, granted=FAKE):
        return lib.dreams_pages_fork_e4m3(ctypes.byref(p), ctypes.byref(s or good()), kp, vp, table, count, kv, ref, n, src,
                                          dst, granted, None)

    eight = lambda **kw: pool(D, **{"dtype": D.DREAMS_E4M3, **kw})
    names = {commit: ("kp", "vp", "table", "kv", "path", "alen", "out"), read: ("kp", "vp", "table", "kv", "ko", "vo"),
             fork: ("kp", "vp", "table", "count", "kv", "ref", "src", "dst", "granted")}
    for f in (commit, read, fork):
        for kw, status in POOLS:
            if kw not in (dict(head_dim=512), dict(page_stride=4100)):
                assert f(eight(**kw)) == status, (f.__name__, kw)
        assert f(pool(D)) == -1 and f(eight(batch=0)) == 0
        for name in names[f]:
            assert f(eight(), **{name: None}) == -1 and f(eight(), **{name: ODD}) == -1, (f.__name__, name)
        for s in (D.PageScales(None, 0x100000, 0, 0), D.PageScales(0x100000, 0x100000, 0, 1),
                  D.PageScales(0x100000, 0x100000, 100, 0)):
            assert f(eight(), s=s) == -1
    assert commit(eight(), ps=0) == -1 and commit(eight(), out=FAKE) == -1
    assert read(eight(), n=-1) == -1 and read(eight(), n=0) == 0 and read(eight(batch=60000)) == -2
    assert read(eight(), n=1 << 30) == -2 and read(eight(), n=(1 << 30) + 1) == -1
    for call, count in ((lib.dreams_paged_kv_commit_e4m3, 6), (lib.dreams_paged_read_e4m3, 4)):
        assert call(ctypes.byref(eight()), None, *[FAKE] * count, 5, *[FAR] * (1 if count == 6 else 2), None) == -1


def test_the_reference_itself():
    """Codes round trip, the nearest one is taken (brute force), and torch's e4m3 agrees."""
    assert np.array_equal(E.encode(E.VALUES[:127]), np.arange(127))
    assert np.nanmax(E.VALUES) == 448 and E.VALUES[1] == 2.0 ** -9
    rng = np.random.default_rng(0)
    x = np.concatenate((rng.uniform(-448, 448, 500), rng.standard_normal(500) * 0.01, (E.VALUES[:126] + E.VALUES[1:127]) / 2))
    got = E.VALUES[E.encode(x)]
    finite = E.VALUES[np.isfinite(E.VALUES)]
    assert (np.abs(got - x) == np.abs(finite[None] - x[:, None]).min(1)).all()
    t = torch.from_numpy(x.astype(np.float32))
    assert np.array_equal(t.to(torch.float8_e4m3fn).double().numpy(), E.VALUES[E.encode(t.double().numpy())])
    for top, s in ((0, 1), (448, 127), (448.0001, 128), (1.75, 119), (3.4e38, 247)):
        assert E.scale_byte(top) == s
    # a rotation by a quarter turn and by none
    x = rng.standard_normal((1, 3, 16))
    one = E.rotate(x, np.array([[0, 1, 2]]), np.full(8, np.pi / 2), 1.0, False)[0]
    assert np.allclose(one[0, 0], x[0, 0]) and np.allclose(one[0, 1], np.concatenate((-x[0, 1, 8:], x[0, 1, :8])))
    two = E.rotate(x, np.array([[0, 1, 2]]), np.full(8, np.pi / 2), 2.0, True)[0]
    assert np.allclose(two[0, 2], -2 * x[0, 2]) and np.allclose(two[0, 1, 0::2], -2 * x[0, 1, 1::2])
