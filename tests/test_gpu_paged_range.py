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


# kind, heads, D, lengths, T or N, window, sinks, splits; workgroups of 128 rows: more than the compute units (256), than two to
# each (512), and in pieces.  Above one to a unit, row groups of one length, and above two, any, have one key group.
MANY = [
    ("prompt", (32, 8), 64, [40] * 17, 70, 0, 0, 1),            # packed: 408 workgroups
    ("prompt", (64, 32), 128, [90] * 9, 67, 0, 0, 1),           # 134 rows a KV head, 576 workgroups
    ("prompt", (16, 16), 64, [0] * 20, 257, 0, 0, 1),           # by heads, no prefix: 960
    ("prompt", (16, 8), 128, [30, 200, 0, 77] * 5, 200, 50, 4, 1),
    ("prompt", (32, 4), 128, [9, 150, 61] * 6, 130, 0, 0, 1),
    ("prompt", (16, 16), 64, [0], 2200, 0, 0, 1),               # 288 groups of 128 to 2200 keys (two key groups)
    ("prompt", (8, 8), 64, [700, 350, 500], 150, 0, 0, 7),      # pieces of fewer groups
    ("prompt", (16, 4), 128, [600, 900, 20], 200, 300, 5, 4),
    ("verify", (40, 20), 64, [120] * 14, 40, 0, 0, 1),          # 80 rows a KV head, 280
    ("verify", (28, 4), 128, [300, 5, 64, 0] * 9, 60, 0, 0, 1), # 576
    ("verify", (32, 8), 64, [90, 33, 0] * 8, 128, 40, 3, 1),
    ("verify", (16, 4), 128, [500, 900, 3], 100, 0, 0, 6),
]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("kind,heads,D,lens,N,window,sinks,splits", MANY)
def test_many_row_groups(dev, kind, heads, D, lens, N, window, sinks, splits, masked):
    """bf16 calls with more workgroups than compute units: two to a unit, a key group each, and their second round.
    (masked: a prompt's ragged rows.)"""
    rng = np.random.default_rng(52)
    Hq, Hkv = heads
    B, G, ps = len(lens), Hq // Hkv, 32
    note("many", kind, heads, D, lens, N, window, sinks, splits, masked)
    rows = G * N
    groups = B * Hkv * -(-rows // 128)     # at least (a head's own groups may be more)
    cus = torch.cuda.get_device_properties(dev).multi_processor_count
    assert rows > 64 and groups * splits > cus and (groups * splits > 2 * cus or splits > 1 or len(set(lens)) == 1)
    q, qh = R.rounded(rng, (B, Hq, N, D), True, dev)
    if kind == "verify":
        c = R.Cache(rng, dev, np.array(lens) + N, Hkv, ps, D, True)
        par = R.tree(rng, B, N)
        see = R.ancestors(par)
        if masked:
            see &= rng.random(see.shape) < 0.6
        out, lse = dreams.paged_verify_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), parent=R.ints(par, dev),
                                            tree_mask=torch.from_numpy(R.mask_bits(see)).to(dev) if masked else None,
                                            window=window, sinks=sinks, num_splits=splits, max_kv_len=max(1, max(lens)))
        torch.cuda.synchronize()
        ref = R.verify(qh, c.k, c.v, c.table, lens, par, see, window, sinks, 1 / np.sqrt(D))
    else:
        live = [int(x) for x in rng.integers(0, N + 1, size=B)] if masked else [N] * B      # (ragged rows)
        width = -(-(max(lens) + N) // ps)
        c = R.Cache(rng, dev, np.array(lens) + np.array(live), Hkv, ps, D, True, width=width)
        for b in range(B):
            q[b, :, live[b]:] = float("nan")
            qh[b, :, live[b]:] = 0
        out, lse = dreams.paged_prompt_attn(q, c.kd, c.vd, c.tabled, R.ints(lens, dev), R.ints(live, dev) if masked else None,
                                            window=window, sinks=sinks, num_splits=splits, max_kv_len=max(1, max(lens)))
        torch.cuda.synchronize()
        ref = R.prompt(qh, c.k, c.v, c.table, lens, live, window, sinks, 1 / np.sqrt(D))
    R.check(out, lse, ref, True, kind)
    size = dreams.paged_verify_attn_workspace_size if kind == "verify" else dreams.paged_prompt_attn_workspace_size
    room = size(dreams.paged_desc(q, c.kd, c.vd, c.tabled, window, sinks, max(1, max(lens)), splits))
    assert room == 0 if splits == 1 else room > 65536 + groups * splits * 128 * D * 4, "pieces"     # (their rows, in fp32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_fork_past_32_bits(dev, dtype):
    """A fork whose partly filled page, and that of the copy, lie more than 2^32 bytes into every layer."""
    bf16, D, ps, Hkv, NL = dtype == "bf16", 128, 64, 2, 2
    dt, size = (torch.bfloat16, 2) if bf16 else (torch.float32, 4)
    rng = np.random.default_rng(53)
    P = (1 << 32) * 5 // 4 // (Hkv * ps * D * size)
    assert P <= dreams.PAGES_MAX and (P - 5) * Hkv * ps * D * size > 1 << 32
    pools = [torch.empty((NL, P, Hkv, ps, D), dtype=dt, device=dev) for _ in range(2)]
    last, copy, rows = P - 3, P - 5, 36
    want = []
    for t in pools:
        for page in (last, copy):
            t[:, page] = R.rounded(rng, (NL, Hkv, ps, D), bf16, dev)[0]
        want.append(t[:, copy].clone())
        want[-1][:, :, :rows] = t[:, last, :, :rows]
    table = R.ints([[P - 1, last, -1], [-1, -1, -1]], dev)
    count, kv_len = R.ints([2, 0], dev), R.ints([ps + rows, 0], dev)
    ref = torch.ones(P, dtype=torch.int32, device=dev)
    ref[copy] = 0
    granted = dreams.pages_fork(*pools, table, count, kv_len, ref, R.ints([0], dev), R.ints([1], dev))
    torch.cuda.synchronize()
    assert granted.tolist() == [1] and table.tolist() == [[P - 1, last, -1], [P - 1, copy, -1]]
    assert count.tolist() == [2, 2] and kv_len.tolist() == [ps + rows] * 2
    assert int(ref[P - 1]) == 2 and int(ref[copy]) == 1 and int(ref.sum()) == P + 1
    for t, w in zip(pools, want):
        assert torch.equal(t[:, copy], w)
