"""Refusals of the paged cache's entry points on the CPU: arguments are checked, with a message, before anything is
enqueued.  No kernel runs here."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def D():
    from paper_2606_00535_amd import dreams
    if not os.path.exists(dreams.LIBRARY):
        from paper_2606_00535_amd import build
        build.build()
    return dreams


FAKE, ODD = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x100002)   # never dereferenced


def desc(D, **kw):
    d = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, num_rows=60, num_pages=100, page_size=16,
             table_width=40, max_kv_len=0, num_splits=1, window=0, sinks=0, dtype=D.DREAMS_BF16, scale=0.088,
             page_stride=0)
    d.update(kw)
    return D.PagedDesc(**d)


BAD = [(dict(batch=-1), -1), (dict(num_q_heads=0), -1), (dict(num_q_heads=7), -1), (dict(num_kv_heads=0), -1),
       (dict(head_dim=96), -2), (dict(num_rows=0), -1), (dict(num_rows=641), -1), (dict(num_pages=0), -1),
       (dict(page_size=0), -1), (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=65536), -2),
       (dict(table_width=0), -1), (dict(table_width=1 << 27), -2), (dict(max_kv_len=-1), -1), (dict(max_kv_len=581), -1),
       (dict(num_splits=-1), -1), (dict(num_splits=5000), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
       (dict(dtype=7), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
       (dict(page_stride=2 * 16 * 128 - 8), -1), (dict(page_stride=2 * 16 * 128 + 4), -1), (dict(page_stride=1 << 50), -1),
       (dict(page_stride=-4096), -1), (dict(batch=1 << 30), -2)]


@pytest.mark.parametrize("kw,status", BAD)
def test_attention_descriptions(D, kw, status):
    n = ctypes.c_size_t(0)
    for f in ("verify", "prompt"):
        size = getattr(D.lib(), "dreams_paged_%s_attn_workspace_size" % f)
        assert size(ctypes.byref(desc(D)), ctypes.byref(n)) == 0
        assert size(ctypes.byref(desc(D, **kw)), ctypes.byref(n)) == status, f
        assert D.lib().dreams_last_error_message().decode() != ""
        assert size(None, ctypes.byref(n)) == -1 and size(ctypes.byref(desc(D)), None) == -1
    assert D.lib().dreams_paged_verify_attn_workspace_size(ctypes.byref(desc(D, num_rows=129)), ctypes.byref(n)) == -1
    assert D.lib().dreams_paged_prompt_attn_workspace_size(ctypes.byref(desc(D, num_rows=129)), ctypes.byref(n)) == 0


def test_attention_calls(D):
    lib = D.lib()

    def verify(d, q=FAKE, k=FAKE, v=FAKE, table=FAKE, kv=FAKE, par=FAKE, mask=None, out=FAKE, lse=FAKE):
        return lib.dreams_paged_verify_attn(ctypes.byref(d), q, k, v, table, kv, par, mask, out, lse, None, 0, None)

    def prompt(d, q=FAKE, k=FAKE, v=FAKE, table=FAKE, kv=FAKE, rows=FAKE, out=FAKE, lse=FAKE):
        return lib.dreams_paged_prompt_attn(ctypes.byref(d), q, k, v, table, kv, rows, out, lse, None, 0, None)

    for f in (verify, prompt):
        assert f(desc(D, batch=0), None, None, None, None, None, None, out=None, lse=None) == 0   # nothing to do
        for name in ("q", "k", "v", "table", "kv", "out"):
            assert f(desc(D), **{name: None}) == -1, name
        for name in ("q", "k", "v", "table", "kv", "out", "lse"):
            assert f(desc(D), **{name: ODD}) == -1, name
    assert verify(desc(D), par=None) == -1 and b"parent or tree_mask" in lib.dreams_last_error_message()
    assert verify(desc(D, window=5), par=None, mask=FAKE) == -1 and b"depths" in lib.dreams_last_error_message()
    assert verify(desc(D), par=ODD) == -1 and verify(desc(D), mask=ctypes.c_void_p(0x100004)) == -1
    assert prompt(desc(D), rows=ODD) == -1
    assert lib.dreams_paged_verify_attn(None, *[FAKE] * 9, None, 0, None) == -1
    assert lib.dreams_paged_prompt_attn(None, *[FAKE] * 8, None, 0, None) == -1


def pool(D, **kw):
    d = dict(num_layers=2, batch=4, num_kv_heads=2, head_dim=128, num_pages=100, page_size=16, table_width=40,
             dtype=D.DREAMS_BF16, layer_stride=0, page_stride=0)
    d.update(kw)
    return D.PagePool(**d)


POOLS = [(dict(num_layers=0), -1), (dict(batch=-1), -1), (dict(num_kv_heads=0), -1), (dict(head_dim=0), -1),
         (dict(head_dim=4), -2), (dict(head_dim=512), -2), (dict(num_pages=0), -1), (dict(page_size=24), -2),
         (dict(table_width=0), -1), (dict(dtype=3), -1), (dict(page_stride=100), -1), (dict(page_stride=4100), -1),
         (dict(layer_stride=4096 * 99), -1), (dict(layer_stride=409604), -1), (dict(layer_stride=-8), -1)]


def test_rows_and_forks(D):
    lib = D.lib()

    def append(p, k=FAKE, v=FAKE, n=5, strides=(4096, 1024, 512, 128), table=FAKE, kv=FAKE, rows=None, kp=FAKE, vp=FAKE):
        st = None if strides is None else (ctypes.c_int64 * 4)(*strides)
        return lib.dreams_paged_append(ctypes.byref(p), k, v, n, st, table, kv, rows, kp, vp, None)

    def commit(p, kp=FAKE, vp=FAKE, table=FAKE, kv=FAKE, path=FAKE, alen=FAKE, ps=60, out=ctypes.c_void_p(0x200000)):
        return lib.dreams_paged_kv_commit(ctypes.byref(p), kp, vp, table, kv, path, alen, ps, out, None)

    def fork(p, kp=FAKE, vp=FAKE, table=FAKE, count=FAKE, kv=FAKE, ref=FAKE, n=2, src=FAKE, dst=FAKE, granted=FAKE):
        return lib.dreams_pages_fork(ctypes.byref(p), kp, vp, table, count, kv, ref, n, src, dst, granted, None)

    for f in (append, commit, fork):
        for kw, status in POOLS:
            assert f(pool(D, **kw)) == status, (f.__name__, kw)
            assert lib.dreams_last_error_message().decode() != ""
        assert f(pool(D, batch=0)) == 0
        for name in ("kp", "vp"):
            assert f(pool(D), **{name: ODD}) == -1
    assert append(pool(D), n=0) == 0 and append(pool(D), n=-1) == -1
    assert append(pool(D), strides=None) == -1
    for bad in ((-8, 1024, 512, 128), (4096, 1028, 512, 128), (4096, 1024, 512, 129), (4096, 1024, 1 << 50, 128)):
        assert append(pool(D), strides=bad) == -1
    assert append(pool(D), n=1 << 30) == -2
    for name in ("k", "v", "table", "kv", "kp", "vp"):
        assert append(pool(D), **{name: None}) == -1 and append(pool(D), **{name: ODD}) == -1
    assert append(pool(D), rows=ODD) == -1
    for name in ("kp", "vp", "table", "kv", "path", "alen", "out"):
        assert commit(pool(D), **{name: None}) == -1 and commit(pool(D), **{name: ODD}) == -1
    assert commit(pool(D), ps=0) == -1
    assert commit(pool(D), out=FAKE) == -1 and b"overlap" in lib.dreams_last_error_message()
    assert fork(pool(D), n=-1) == -1 and fork(pool(D), n=0) == 0 and fork(pool(D), n=4097) == -2
    assert fork(pool(D, num_pages=524289)) == -2 and fork(pool(D, batch=4097)) == -2
    for name in ("kp", "vp", "table", "count", "kv", "ref", "src", "dst", "granted"):
        assert fork(pool(D), **{name: None}) == -1 and fork(pool(D), **{name: ODD}) == -1
    assert append(pool(D, num_layers=70000)) == -2 and append(pool(D, batch=70000)) == -2


def test_reserve_and_release(D):
    lib = D.lib()

    def reserve(p, table=FAKE, count=FAKE, ref=FAKE, want=FAKE, granted=FAKE):
        return lib.dreams_pages_reserve(ctypes.byref(p), table, count, ref, want, granted, None)

    def release(p, table=FAKE, count=FAKE, kv=FAKE, ref=FAKE, n=2, seqs=FAKE, trim=0):
        return lib.dreams_pages_release(ctypes.byref(p), table, count, kv, ref, n, seqs, trim, None)

    for f in (reserve, release):
        for kw, status in ((dict(batch=-1), -1), (dict(num_pages=0), -1), (dict(num_pages=524289), -2),
                           (dict(batch=4097), -2), (dict(page_size=20), -2), (dict(table_width=0), -1),
                           (dict(batch=4096, table_width=1 << 20), -2), (dict(table_width=1 << 27), -2)):
            assert f(pool(D, **kw)) == status, (f.__name__, kw)
        assert f(pool(D, batch=0)) == 0
        for name in ("table", "count", "ref"):
            assert f(pool(D), **{name: None}) == -1 and f(pool(D), **{name: ODD}) == -1
    for name in ("want", "granted"):
        assert reserve(pool(D), **{name: None}) == -1 and reserve(pool(D), **{name: ODD}) == -1
    for name in ("kv", "seqs"):
        assert release(pool(D), **{name: None}) == -1 and release(pool(D), **{name: ODD}) == -1
    assert release(pool(D), trim=2) == -1 and release(pool(D), n=-1) == -1 and release(pool(D), n=0) == 0
    assert release(pool(D), n=4097) == -2
    assert lib.dreams_pages_reserve(None, *[FAKE] * 5, None) == -1
    assert lib.dreams_pages_release(None, *[FAKE] * 4, 1, FAKE, 0, None) == -1


def test_bindings(D):
    """Wrong types, host tensors and layouts are refused before anything else (no GPU needed)."""
    q = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    table, one = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        D.paged_verify_attn(q, pages, pages, table, one, parent=torch.zeros((1, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="device tensor"):
        D.paged_prompt_attn(q, pages, pages, table, one)
    with pytest.raises(TypeError):
        D.paged_prompt_attn(q, None, pages, table, one)
    with pytest.raises(ValueError, match="device tensor"):
        D.paged_append(q, q, pages, pages, table, one)
    with pytest.raises(ValueError, match="device tensor"):
        D.paged_kv_commit(pages, pages, table, one, table, one)
    with pytest.raises(ValueError, match="device tensor"):
        D.pages_reserve(table, one, torch.zeros(4, dtype=torch.int32), one, 16)
    with pytest.raises(TypeError, match="int32"):
        D.pages_reserve(table.long(), one, torch.zeros(4, dtype=torch.int32), one, 16)
    with pytest.raises(ValueError, match="device tensor"):
        D.pages_fork(pages, pages, table, one, one, torch.zeros(4, dtype=torch.int32), one, one)
    with pytest.raises(ValueError, match="device tensor"):
        D.pages_release(table, one, one, torch.zeros(4, dtype=torch.int32), one, 16)


def test_limits_of_a_launch(D):
    """Calls with more threads than a launch can have are refused by name."""
    n = ctypes.c_size_t(0)
    big = dict(batch=1 << 10, num_q_heads=32, num_kv_heads=8, page_size=1024, table_width=1024)
    size = D.lib().dreams_paged_prompt_attn_workspace_size
    # 2^15 heads of 4096 rows: 2^25 workgroups of 1024 threads in fp32, 2^20 of 128 rows in bf16
    assert size(ctypes.byref(desc(D, num_rows=4096, dtype=D.DREAMS_F32, **big)), ctypes.byref(n)) == -2
    assert size(ctypes.byref(desc(D, num_rows=4096, **big)), ctypes.byref(n)) == 0
    assert size(ctypes.byref(desc(D, num_rows=511, dtype=D.DREAMS_F32, **big)), ctypes.byref(n)) == 0
    # 2^27 units of one row group
    assert size(ctypes.byref(desc(D, batch=1 << 24, num_q_heads=8, num_kv_heads=8, num_rows=1)), ctypes.byref(n)) == -2
    pool = D.PagePool(1, 1, 8, 128, 4, 16, 4, D.DREAMS_BF16, 0, 0)
    strides = (ctypes.c_int64 * 4)(0, 0, 128, 1024)
    append = lambda rows: D.lib().dreams_paged_append(ctypes.byref(pool), None, None, rows, strides, FAKE, FAKE, None,
                                                      FAKE, FAKE, None)
    assert append(1 << 25) == -2             # 2^25 rows of 8 heads, 16 words each: 2^32 threads
    assert append((1 << 25) - 2) == -1       # (it fits: the next check, of k_new, refuses it)
    wide = D.PagePool(60000, 60000, 8, 64, 4, 16, 4, D.DREAMS_BF16, 0, 0)
    assert D.lib().dreams_paged_kv_commit(ctypes.byref(wide), *[FAKE] * 6, 5, FAKE, None) == -2


def test_views_whose_pages_share_memory(D):
    """An expanded view has no stride between its pages (or layers): refused, not taken for a dense pool."""
    table, one = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    page, layer = torch.zeros((1, 2, 16, 64)), torch.zeros((1, 4, 2, 16, 64))
    for pages in (page.expand(4, 2, 16, 64), layer.expand(3, 4, 2, 16, 64)):
        with pytest.raises(ValueError, match="share memory"):
            D.paged_append(pages, pages, pages, pages, table, one)
        with pytest.raises(ValueError, match="share memory"):
            D.paged_kv_commit(pages, pages, table, one, table, one)
        with pytest.raises(ValueError, match="share memory"):
            D.pages_fork(pages, pages, table, one, one, torch.zeros(4, dtype=torch.int32), one, one)
    with pytest.raises(ValueError, match="share memory"):
        D.paged_prompt_attn(torch.zeros((1, 2, 3, 64)), page.expand(4, 2, 16, 64), page.expand(4, 2, 16, 64), table, one)
    with pytest.raises(ValueError, match="device tensor"):    # (one page, one layer: no stride is used)
        D.paged_append(page, page, page.expand(1, 2, 16, 64), page, table, one)
