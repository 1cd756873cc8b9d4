"""Timed cases of the paged cache: attention over pages, the rows that go into them, and their bookkeeping.

A pool of pages holds every sequence's keys and values, [pages, KV heads, slots, head_dim] a layer; a table names the
pages of a sequence in slot order.  The kinds of call are

    verify   one layer's tree attention over pages (one node: a single token), with or without a sliding window
             behind which only the first tokens stay in sight
    prompt   one layer's causal attention of a prompt, or of a piece of one behind a cached prefix
    rows     a step's new rows written into every layer's pages, then the accepted path compacted there
    pages    sequences dropped, others forked in their place, and room made for the next step's rows

``listed()`` names the cases that stand for the range, ``draw()`` gives others of the same range.  Where ``own`` is
false, ``run`` computes them in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda"


def _dreams():
    from paper_2606_00535_amd import dreams
    return dreams


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # single tokens of a few long sequences, window and sinks: the launch and the latency of the reads count
        dict(name="verify_token_sinks", kind="verify", dtype="bf16", batch=4, hq=32, hkv=8, d=128, lo=1500, hi=8192,
             nodes=1, depth=0, branch=1, page=16, window=1024, sinks=4, mask=False, paired=False),
        # the fp32 model with options: mask bits, ragged lengths, head_dim 64, grouped heads, K and V in one pool
        dict(name="verify_f32_mask", kind="verify", dtype="f32", batch=2, hq=8, hkv=4, d=64, lo=201, hi=640, nodes=16,
             depth=4, branch=3, page=16, window=300, sinks=5, mask=True, paired=True),
        # an ordinary step at batch 1: one LLaVA-1.6-7B layer, 2880 image and 256 text tokens, a 60-node tree
        dict(name="verify_7b_layer", kind="verify", dtype="bf16", batch=1, hq=32, hkv=32, d=128, lo=3136, hi=3136,
             nodes=60, depth=6, branch=4, page=64, window=0, sinks=0, mask=False, paired=False),
        # many long sequences over few KV heads and wide trees: the matrix cores' case
        dict(name="verify_gqa_long", kind="verify", dtype="bf16", batch=16, hq=28, hkv=4, d=128, lo=8192, hi=8192,
             nodes=128, depth=8, branch=6, page=32, window=0, sinks=0, mask=False, paired=False),
        # short prompts of a padded batch, no prefix
        dict(name="prompt_short_ragged", kind="prompt", dtype="bf16", batch=8, hq=24, hkv=8, d=64, lo=0, hi=0, rlo=1,
             rows=187, page=16, window=0, sinks=0, paired=False),
        # a LLaVA-1.6-7B prompt: 2880 image and 256 text tokens
        dict(name="prompt_7b", kind="prompt", dtype="bf16", batch=1, hq=32, hkv=32, d=128, lo=0, hi=0, rlo=3136,
             rows=3136, page=64, window=0, sinks=0, paired=False),
        # pieces of long prompts behind what is cached of them, in a layer with a window
        dict(name="prompt_piece_sinks", kind="prompt", dtype="bf16", batch=2, hq=32, hkv=8, d=128, lo=2900, hi=6400,
             rlo=700, rows=1000, page=32, window=1024, sinks=4, paired=True),
        # a long prompt over few KV heads: the largest product
        dict(name="prompt_gqa_long", kind="prompt", dtype="bf16", batch=1, hq=28, hkv=4, d=128, lo=0, hi=0, rlo=8192,
             rows=8192, page=64, window=0, sinks=0, paired=False),
        # the fp32 model's step: one layer, one sequence
        dict(name="rows_tiny_f32", kind="rows", dtype="f32", layers=1, batch=1, hkv=4, d=64, lo=640, hi=640, nodes=16,
             depth=4, branch=3, page=16, paired=False),
        # a LLaVA-1.6-7B step of four sequences: 32 layers' rows in and compacted
        dict(name="rows_7b_b4", kind="rows", dtype="bf16", layers=32, batch=4, hkv=32, d=128, lo=500, hi=800, nodes=60,
             depth=6, branch=4, page=64, paired=False),
        # one sequence forked in a small pool: the bookkeeping alone
        dict(name="pages_one", kind="pages", dtype="bf16", layers=1, batch=2, forks=1, hkv=4, d=128, lo=500, hi=900,
             page=16, extra=60, spare=64, paired=False),
        # six of eight sequences replaced by forks of the other two, 32 layers
        dict(name="pages_beams", kind="pages", dtype="bf16", layers=32, batch=8, forks=6, hkv=4, d=128, lo=1000, hi=2900,
             page=32, extra=128, spare=128, paired=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _tree_shape(rng, most):
    nodes = 1 if rng.random() < 0.2 else _log_int(rng, 1, most)
    depth = rng.randint(min(3, nodes - 1), min(8, nodes - 1)) if nodes > 1 else 0
    return dict(nodes=nodes, depth=depth, branch=rng.randint(4, 6) if nodes <= 60 else 6)


def _window(rng, hi):
    if rng.random() < 0.5:
        return dict(window=0, sinks=0)
    return dict(window=_log_int(rng, 1, max(2, hi)), sinks=rng.choice((0, 1, 4, 17, 64)))


_HEADS = ((32, 32), (40, 40), (28, 4), (32, 8), (24, 8), (16, 16), (8, 2), (7, 1))
_PAGES = (16, 16, 32, 64, 128, 256)


def draw(rng):
    """One more case of the listed kinds, its sizes spread over the range that they cover."""
    kind = rng.choice(("verify", "verify", "verify", "verify_f32", "prompt", "prompt", "prompt", "rows", "pages"))
    common = dict(page=rng.choice(_PAGES), paired=rng.random() < 0.3)
    if kind == "verify":
        hq, hkv = rng.choice(_HEADS)
        hi = _log_int(rng, 1, 8192)
        batch = min(_log_int(rng, 1, 16), max(1, 16 * 4 * 8192 // (hkv * hi)))
        return dict(kind="verify", dtype="bf16", batch=batch, hq=hq, hkv=hkv, d=rng.choice((64, 128, 128)),
                    lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi, mask=rng.random() < 0.3, **_window(rng, hi),
                    **_tree_shape(rng, 128), **common)
    if kind == "verify_f32":
        hq, hkv = rng.choice(((4, 4), (4, 2), (6, 2), (3, 3), (8, 8)))
        hi = _log_int(rng, 1, 1300)
        return dict(kind="verify", dtype="f32", batch=rng.randint(1, 2), hq=hq, hkv=hkv, d=rng.choice((64, 128)),
                    lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi, mask=rng.random() < 0.3, **_window(rng, hi),
                    **_tree_shape(rng, 100), **common)
    if kind == "prompt":
        hq, hkv = rng.choice(((32, 32), (28, 4), (32, 8), (24, 8), (8, 2), (7, 1)))
        rows = _log_int(rng, 1, 8192)
        hi = 0 if rng.random() < 0.5 else _log_int(rng, 1, 8192)
        most = 28 * 8192 * 4096     # the longest listed prompt's scores
        if hq * rows * (hi + rows / 2) > most:
            hi = 0
        if hq * rows * rows / 2 > most:
            hq, hkv = 28, 4
        batch = max(1, min(rng.randint(1, 8), int(most / (hq * rows * (hi + rows / 2)))))
        dtype = "f32" if hq * batch * rows * (hi + rows) < 3e7 and rng.random() < 0.4 else "bf16"
        return dict(kind="prompt", dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=rng.choice((64, 128, 128)),
                    lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi, rlo=int(rows * rng.uniform(0.0, 1.0)), rows=rows,
                    **_window(rng, hi + rows), **common)
    hkv, d, dtype = rng.choice((1, 2, 4, 8, 16)), rng.choice((64, 128)), rng.choice(("bf16", "bf16", "f32"))
    size = 4 if dtype == "f32" else 2
    if kind == "rows":
        hi, batch = _log_int(rng, 1, 2900), rng.randint(1, 4)
        most = max(1, min(32, 10 ** 9 // (batch * (hi + 128) * hkv * d * size * 2)))     # (a pool of a gigabyte)
        return dict(kind="rows", dtype=dtype, layers=_log_int(rng, 1, most), batch=batch, hkv=hkv, d=d,
                    lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi, **_tree_shape(rng, 128), **common)
    hi, batch, spare = _log_int(rng, 1, 8192), rng.randint(2, 8), _log_int(rng, 8, 512)
    slots = batch * (hi + 128) + (spare + 3 * batch) * common["page"]
    most = max(1, min(32, 10 ** 9 // (slots * hkv * d * size * 2)))
    return dict(kind="pages", dtype=dtype, layers=_log_int(rng, 1, most), batch=batch, forks=rng.randint(1, batch - 1),
                hkv=hkv, d=d, lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi, extra=rng.randint(1, 128), spare=spare,
                **common)


# ------------------------------------------------------------------------------------------------------- inputs
class _Inputs:
    """Seeded draws on the device (tensors) and the host (trees, lengths, tables)."""

    def __init__(self, case, seed):
        self.host = np.random.default_rng(seed)
        self.gen = torch.Generator(device=DEVICE)
        self.gen.manual_seed(int(seed))
        self.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def normal(self, shape, std=1.0):
        return torch.empty(shape, dtype=self.dtype, device=DEVICE).normal_(0.0, std, generator=self.gen)

    def lengths(self, lo, hi, batch):
        """Lengths lo..hi, the longest one present (a server sizes its bound by it)."""
        n = self.host.integers(lo, hi + 1, size=batch).astype(np.int32)
        n[int(self.host.integers(batch))] = hi
        return n

    def pool(self, lead, pages, case):
        """(k, v) pools: two tensors, or the two halves of every page of one."""
        tail = (case["hkv"], case["page"], case["d"])
        if case["paired"]:
            both = self.normal(lead + (pages, 2) + tail)
            return both.select(len(lead) + 1, 0), both.select(len(lead) + 1, 1)
        return self.normal(lead + (pages,) + tail), self.normal(lead + (pages,) + tail)

    def table(self, counts, width, pages):
        """Every sequence's pages from anywhere in the pool, as after some time of service; -1 past them."""
        ids = self.host.permutation(pages).astype(np.int32)
        table = np.full((len(counts), width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(counts):
            table[b, :n] = ids[at:at + n]
            at += n
        return table

    def trees(self, case):
        return np.stack([_tree(self.host, case["nodes"], case["depth"], case["branch"])
                         for _ in range(case["batch"])])


def _tree(host, nodes, depth, branch):
    """A parent array in breadth-first order: a spine of `depth` nodes, the others anywhere above that depth."""
    up, deep, kids = [-1], [0], [0]
    while len(up) < nodes:
        n = len(up)
        if n <= depth:
            p = n - 1
        else:
            free = [i for i in range(n) if deep[i] < depth and kids[i] < branch]
            p = free[int(host.integers(len(free)))]
        up.append(p)
        deep.append(deep[p] + 1)
        kids.append(0)
        kids[p] += 1
    order = sorted(range(nodes), key=lambda i: deep[i])     # stable: children behind their parents
    place = {i: n for n, i in enumerate(order)}
    return np.array([-1 if up[i] < 0 else place[up[i]] for i in order], dtype=np.int32)


def _device(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)


def _depths(parent):
    deep = np.zeros(parent.shape, dtype=np.int32)
    for b in range(parent.shape[0]):
        for i in range(1, parent.shape[1]):
            deep[b, i] = deep[b, parent[b, i]] + 1
    return deep


def _ancestors(parent):
    """[B, T, T] truth values: node j is node i or an ancestor of it."""
    batch, nodes = parent.shape
    see = np.zeros((batch, nodes, nodes), dtype=bool)
    for b in range(batch):
        for i in range(nodes):
            if i:
                see[b, i] = see[b, parent[b, i]]
            see[b, i, i] = True
    return see


def _mask_bits(see):
    batch, nodes, _ = see.shape
    words = (nodes + 63) // 64
    bits = np.zeros((batch, nodes, words * 64), dtype=np.uint8)
    bits[:, :, :nodes] = see
    return np.packbits(bits, axis=2, bitorder="little").view(np.int64).reshape(batch, nodes, words)


def _prepare_verify(case, seed):
    r = _Inputs(case, seed)
    batch, nodes, page = case["batch"], case["nodes"], case["page"]
    lengths, parent = r.lengths(case["lo"], case["hi"], batch), r.trees(case)
    counts, width = -(-(lengths + nodes) // page), -(-(case["hi"] + nodes) // page)
    pages = batch * width + 3
    see, deep = _ancestors(parent), _depths(parent)
    if case["mask"]:
        see &= r.host.random(see.shape) < 0.7   # a caller's own mask: some ancestors hidden, now and then all of a row
    k, v = r.pool((), pages, case)
    q = r.normal((batch, case["hq"], nodes, case["d"]), 0.125 if case["dtype"] == "f32" else 1.0)
    return dict(kind="verify", case=case, lengths=lengths, q=q, k=k, v=v, table=_device(r.table(counts, width, pages)),
                kv_len=_device(lengths), parent=_device(parent), see=_device(see), deep=_device(deep),
                mask=_device(_mask_bits(see)) if case["mask"] else None)


def _prepare_prompt(case, seed):
    r = _Inputs(case, seed)
    batch, page = case["batch"], case["page"]
    lengths, rows = r.lengths(case["lo"], case["hi"], batch), r.lengths(case["rlo"], case["rows"], batch)
    counts = -(-(lengths + rows) // page)
    # a table wide enough for the padded rows of the longest prefix, as a server sizes it
    width = -(-(case["hi"] + case["rows"]) // page)
    pages = batch * width + 3
    k, v = r.pool((), pages, case)
    return dict(kind="prompt", case=case, lengths=lengths, rows=rows, k=k, v=v,
                q=r.normal((batch, case["hq"], case["rows"], case["d"])),
                table=_device(r.table(counts, width, pages)), kv_len=_device(lengths), row_len=_device(rows))


def _prepare_rows(case, seed):
    r = _Inputs(case, seed)
    batch, nodes, page = case["batch"], case["nodes"], case["page"]
    lengths, parent = r.lengths(case["lo"], case["hi"], batch), r.trees(case)
    counts, width = -(-(lengths + nodes) // page), -(-(case["hi"] + nodes) // page)
    pages = batch * width + 3
    deep = _depths(parent)
    path = np.full((batch, nodes), -1, dtype=np.int32)
    taken = np.zeros(batch, dtype=np.int32)
    for b in range(batch):      # the way from the root to some node
        i = int(r.host.integers(nodes))
        taken[b] = deep[b, i]
        while i >= 0:
            path[b, deep[b, i]] = i
            i = int(parent[b, i])
    k, v = r.pool((case["layers"],), pages, case)
    # a projection's output: token by token, a token's heads side by side
    new = (case["layers"], batch, nodes, case["hkv"], case["d"])
    return dict(kind="rows", case=case, lengths=lengths, taken=taken, k=k, v=v,
                k_new=r.normal(new).transpose(2, 3), v_new=r.normal(new).transpose(2, 3),
                table=_device(r.table(counts, width, pages)), kv_len=_device(lengths), path=_device(path),
                accepted=_device(taken))


def _prepare_pages(case, seed):
    r = _Inputs(case, seed)
    batch, page, forks = case["batch"], case["page"], case["forks"]
    lengths = r.lengths(case["lo"], case["hi"], batch)
    counts = -(-lengths // page)
    width = -(-(case["hi"] + case["extra"]) // page) + 1
    pages = batch * width + case["spare"]
    table = r.table(counts, width, pages)
    held = np.zeros(pages, dtype=np.int32)
    held[table[table >= 0]] = 1
    order = r.host.permutation(batch).astype(np.int32)
    dst, kept = np.sort(order[:forks]), order[forks:]
    src = kept[r.host.integers(len(kept), size=forks)]
    after = lengths.copy()
    after[dst] = lengths[src]
    k, v = r.pool((case["layers"],), pages, case)
    return dict(kind="pages", case=case, k=k, v=v, table=_device(table), count=_device(counts.astype(np.int32)),
                kv_len=_device(lengths), refcount=_device(held), src=_device(src), dst=_device(dst),
                want=_device((after + case["extra"]).astype(np.int32)))


def prepare(case, seed):
    return globals()["_prepare_" + case["kind"]](case, seed)


# ------------------------------------------------------------------------------------- the framework's operators
def _own_verify(s):
    case = s["case"]
    return _dreams().paged_verify_attn(s["q"], s["k"], s["v"], s["table"], s["kv_len"], parent=s["parent"],
                                       tree_mask=s["mask"], window=case["window"], sinks=case["sinks"],
                                       max_kv_len=case["hi"])


def _own_prompt(s):
    case = s["case"]
    return _dreams().paged_prompt_attn(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["row_len"],
                                       window=case["window"], sinks=case["sinks"], max_kv_len=case["hi"])


def _own_rows(s):
    dreams = _dreams()
    dreams.paged_append(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["kv_len"])
    kept = dreams.paged_kv_commit(s["k"], s["v"], s["table"], s["kv_len"], s["path"], s["accepted"])
    return dict(k=s["k"], v=s["v"], kv_len=kept)


def _own_pages(s):
    dreams, page = _dreams(), s["case"]["page"]
    dreams.pages_release(s["table"], s["count"], s["kv_len"], s["refcount"], s["dst"], page)
    forked = dreams.pages_fork(s["k"], s["v"], s["table"], s["count"], s["kv_len"], s["refcount"], s["src"], s["dst"])
    room = dreams.pages_reserve(s["table"], s["count"], s["refcount"], s["want"], page)
    return dict(forked=forked, room=room, table=s["table"], count=s["count"], kv_len=s["kv_len"],
                refcount=s["refcount"], k=s["k"], v=s["v"])


# ------------------------------------------------------------------------------------------------ the plain forms
def _rows_of(pool, pages, n):
    """The first n slots that a sequence's pages hold: [KV heads, n, D], in 32 bits."""
    x = pool[pages.long()].float()                      # [pages, KV heads, slots, D]
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :n].contiguous()


def _attend(q, k, v, see):
    """softmax over the keys in sight; q [heads, rows, D], k and v [heads, keys, D], see [rows, keys] (rows of a head
    group after one another).  A row that sees nothing: 0 and -inf."""
    z = torch.matmul(q * (1.0 / math.sqrt(q.shape[2])), k.transpose(1, 2).contiguous())
    z = z.masked_fill(~see, -math.inf)
    top = z.amax(dim=2, keepdim=True)
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(dim=2, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return out, (top + torch.log(total))[:, :, 0]


def _in_sight(where, keys, case):
    """[rows, keys]: position `where` of a row against position `keys` of a key."""
    if case["window"] == 0:
        return torch.ones((len(where), len(keys)), dtype=torch.bool, device=DEVICE)
    return (where[:, None] - keys[None, :] < case["window"]) | (keys[None, :] < case["sinks"])


def _plain_verify(s):
    case, q = s["case"], s["q"]
    batch, hq, nodes, d = q.shape
    hkv = case["hkv"]
    out, lse = torch.empty_like(q), torch.empty((batch, hq, nodes), device=DEVICE)
    for b in range(batch):
        n = int(s["lengths"][b])
        pages = s["table"][b, :-(-(n + nodes) // case["page"])]
        k, v = _rows_of(s["k"], pages, n + nodes), _rows_of(s["v"], pages, n + nodes)
        where = n + s["deep"][b]
        at = torch.cat((torch.arange(n, device=DEVICE, dtype=torch.int32), where))
        see = torch.cat((torch.ones((nodes, n), dtype=torch.bool, device=DEVICE), s["see"][b]), dim=1)
        see = (see & _in_sight(where, at, case)).repeat(hq // hkv, 1)
        x, y = _attend(q[b].float().reshape(hkv, -1, d), k, v, see)
        out[b], lse[b] = x.reshape(hq, nodes, d).to(q.dtype), y.reshape(hq, nodes)
    return out, lse


def _plain_prompt(s):
    case, q = s["case"], s["q"]
    batch, hq, rows, d = q.shape
    hkv = case["hkv"]
    group = hq // hkv
    out, lse = torch.zeros_like(q), torch.full((batch, hq, rows), -math.inf, device=DEVICE)
    for b in range(batch):
        n, m = int(s["lengths"][b]), int(s["rows"][b])
        if m == 0:
            continue
        pages = s["table"][b, :-(-(n + m) // case["page"])]
        k, v = _rows_of(s["k"], pages, n + m), _rows_of(s["v"], pages, n + m)
        where, at = n + torch.arange(m, device=DEVICE), torch.arange(n + m, device=DEVICE)
        see = (at[None, :] <= where[:, None]) & _in_sight(where, at, case)
        step = max(1, 2 ** 28 // (m * (n + m)))      # heads at a time: the scores of a long prompt are large
        for h in range(0, hq, step):
            of = torch.arange(h, min(h + step, hq), device=DEVICE) // group
            x, y = _attend(q[b, h:h + step, :m].float(), k[of], v[of], see)
            out[b, h:h + step, :m], lse[b, h:h + step, :m] = x.to(q.dtype), y
    return out, lse


def _plain_rows(s):
    case = s["case"]
    nodes, page = case["nodes"], case["page"]
    for b in range(case["batch"]):
        n, a = int(s["lengths"][b]), int(s["taken"][b])
        slot = n + torch.arange(nodes, device=DEVICE)
        ids, row = s["table"][b].long()[slot // page], slot % page
        for pool, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
            pool[:, ids, :, row] = new[:, b].permute(2, 0, 1, 3)    # [nodes, layers, KV heads, D]
            way = s["path"][b, :a + 1].long()
            pool[:, ids[:a + 1], :, row[:a + 1]] = pool[:, ids[way], :, row[way]]
    return dict(k=s["k"], v=s["v"], kv_len=s["kv_len"] + s["accepted"] + 1)


def _lowest_free(refcount, need):
    """Sequences in order, each granted if as many pages as it needs are free; the pages, lowest first.
    Returns (granted [n] int32, first [n]: where a granted one's pages begin in the order of the free ones, order)."""
    free = (refcount == 0).long()
    left = free.sum()
    granted, first, used = [], [], torch.zeros_like(left)
    for want in need.long().unbind():
        ok = (want <= left - used).long()
        granted.append(ok)
        first.append(used)
        used = used + want * ok
    rank = torch.cumsum(free, 0) - 1
    order = torch.zeros(len(refcount) + 1, dtype=torch.long, device=DEVICE)
    order.scatter_(0, torch.where(free == 1, rank, torch.full_like(rank, len(refcount))),
                   torch.arange(len(refcount), device=DEVICE))
    return torch.stack(granted).int(), torch.stack(first), order


def _plain_pages(s):
    case, table, count, lens, refcount = s["case"], s["table"], s["count"], s["kv_len"], s["refcount"]
    page, src, dst = case["page"], s["src"].long(), s["dst"].long()
    width = table.shape[1]
    column = torch.arange(width, device=DEVICE)
    slots = torch.zeros(len(refcount) + 1, dtype=torch.int32, device=DEVICE)

    def add(ids, by):       # page id -1: nowhere
        slots.zero_()
        slots.scatter_add_(0, torch.where(ids < 0, torch.full_like(ids, len(refcount)), ids).long().reshape(-1),
                           torch.full_like(ids, by).reshape(-1))
        refcount.add_(slots[:-1])

    # drop the sequences that are replaced
    add(table[dst], -1)
    table[dst] = -1
    count[dst] = 0
    lens[dst] = 0
    # fork: whole pages shared, the partly filled one copied
    n = lens[src]
    whole, tail = n // page, n % page
    granted, first, order = _lowest_free(refcount, (tail > 0).int())
    shared = torch.where((column[None, :] < whole[:, None]) & (granted[:, None] == 1), table[src],
                         torch.full_like(table[src], -1))
    add(shared, 1)
    fresh = order[first].int()
    copied = (granted == 1) & (tail > 0)
    old = table[src].gather(1, whole.clamp(max=width - 1).long()[:, None])[:, 0]
    table[dst] = torch.where((column[None, :] == whole[:, None]) & copied[:, None], fresh[:, None], shared)
    add(torch.where(copied, fresh, torch.full_like(fresh, -1)), 1)
    count[dst] = (whole + copied.int()) * granted
    lens[dst] = n * granted
    for i in range(case["forks"]):
        for pool in (s["k"], s["v"]):
            was = pool[:, old[i].clamp(min=0).long()]
            to = fresh[i].long()[None]
            keep = (torch.arange(page, device=DEVICE) < tail[i])[None, None, :, None] & copied[i]
            pool[:, to] = torch.where(keep, was, pool[:, to][:, 0])[:, None]
    # room for the next rows
    need = ((s["want"] + page - 1) // page - count).clamp(min=0)
    room, first, order = _lowest_free(refcount, need)
    at = column[None, :] - count[:, None]
    new = (at >= 0) & (at < need[:, None]) & (room[:, None] == 1)
    ids = order[(first[:, None] + at).clamp(min=0, max=len(refcount))].int()
    table.copy_(torch.where(new, ids, table))
    add(torch.where(new, ids, torch.full_like(ids, -1)), 1)
    count.add_(need * room)
    return dict(forked=granted, room=room, table=table, count=count, kv_len=lens, refcount=refcount, k=s["k"],
                v=s["v"])


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["kind"]](state)


# ------------------------------------------------------------------------------------------------- what it takes
def _seen(where, window, sinks):
    """Keys at positions up to `where` that a row there sees (an array of positions)."""
    every = where + 1.0
    if window == 0:
        return every
    near = np.minimum(every, window)
    return near + np.minimum(np.maximum(every - near, 0), sinks)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    d, hkv = case["d"], case["hkv"]
    if case["kind"] in ("verify", "prompt"):
        window, sinks, prefix = case["window"], case["sinks"], (case["lo"] + case["hi"]) / 2
        if case["kind"] == "verify":
            rows = case["nodes"]
            seen = float(_seen(np.array([prefix]), window, sinks)[0]) * rows + rows * case["depth"] / 2
            keys = float(_seen(np.array([prefix]), window, sinks)[0]) + rows - 1
        else:
            rows = (case["rlo"] + case["rows"]) / 2
            at = _seen(prefix + np.arange(max(int(rows), 1)), window, sinks)
            seen = float(at.sum())
            keys = min(prefix + rows, float(at[0]) + rows)
        heads = case["batch"] * case["hq"]
        moved = 2 * case["batch"] * hkv * keys * d * size + 2 * heads * rows * d * size + heads * rows * 4
        return dict(bytes=moved, flops=4.0 * heads * seen * d)
    row = hkv * d * size * 2 * case["layers"]      # a slot's K and V in every layer
    if case["kind"] == "rows":
        return dict(bytes=2.0 * row * case["batch"] * (case["nodes"] + case["depth"] / 2), flops=0)
    tail = (case["page"] - 1) / 2 if case["page"] <= case["hi"] else case["hi"] / 2
    tables = case["batch"] * (-(-(case["hi"] + case["extra"]) // case["page"]) + 4) * 4
    return dict(bytes=2.0 * row * case["forks"] * tail + 2.0 * tables, flops=0)


# --------------------------------------------------------------------------------------- the same, in 64 bits
def _softmax64(scores, values):
    """(out, lse) of one head's masked scores [rows, keys] in 64 bits."""
    lse = torch.logsumexp(scores, dim=1)
    p = torch.exp(scores - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    return p @ values, lse


def exact(case, seed):
    """Row by row of the definition: every slot's place looked up in the table, every key's place compared with the
    row's.  Bookkeeping and copies have no value in 64 bits."""
    if case["kind"] in ("rows", "pages"):
        return None
    s = prepare(case, seed)
    q, page, table = s["q"], case["page"], s["table"].cpu().numpy()
    batch, hq, rows, d = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full((batch, hq, rows), -math.inf, dtype=torch.float64, device=DEVICE)
    for b in range(batch):
        n = int(s["lengths"][b])
        m = rows if case["kind"] == "verify" else int(s["rows"][b])
        if m == 0:
            continue
        slots = np.arange(n + m)
        ids, place = _device(table[b][slots // page].astype(np.int64)), _device(slots % page)
        if case["kind"] == "verify":
            depth = s["deep"][b].cpu().numpy()
            row_at, key_at = n + depth, np.concatenate((np.arange(n), n + depth))
            sight = np.ones((m, n + m), dtype=bool)
            sight[:, n:] = s["see"][b].cpu().numpy()
        else:
            row_at, key_at = n + np.arange(m), slots
            sight = key_at[None, :] <= row_at[:, None]
        if case["window"]:
            sight &= (key_at[None, :] < case["sinks"]) | (row_at[:, None] - key_at[None, :] < case["window"])
        hidden = _device(~sight)
        for g in range(case["hkv"]):
            keys, values = s["k"][ids, g, place].double(), s["v"][ids, g, place].double()
            for h in range(g * hq // case["hkv"], (g + 1) * hq // case["hkv"]):
                z = q[b, h, :m].double() @ keys.t().contiguous() / math.sqrt(d)
                out[b, h, :m], lse[b, h, :m] = _softmax64(z.masked_fill_(hidden, -math.inf), values)
    return out, lse
