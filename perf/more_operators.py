"""Timed cases of positions and of a cache in 8 bits: rotary positions, rotated rows on their way into pages, pages of
e4m3 values with a power-of-two scale for each 16 slots of a head, and the attention over them.

A rotation turns a pair of a head's columns by its position times the pair's frequency.  Pages of 8 bits are
[pages, KV heads, slots, head_dim] in e4m3, their scales [pages, KV heads, slots / 16] in e8m0: a slot's row is its codes times
2^(scale - 127).  A block of 16 slots takes the least scale at which its largest value is at most 448, e4m3's largest; rows
that it holds already keep theirs or move to a larger one with it.  The kinds of call are

    turn      queries or keys of consecutive, drafted or given positions rotated
    append    a step's or prompt's queries rotated, its keys rotated into their pages, its values put beside them
    store8    the same into pages of 8 bits; of a draft tree, the accepted path is compacted there; the cache is read back
    verify8   one layer's tree attention over pages of 8 bits (one node: a single token), with or without a window
    prompt8   one layer's causal attention of a prompt, or of a piece of one behind a cached prefix, over the same

``listed()`` names the cases that stand for the range, ``draw()`` gives others of the same range.  Where ``own`` is
false, ``run`` computes them in elementary torch operations in 32 bits (angles in 64).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda"
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _dreams():
    from paper_2606_00535_amd import dreams
    return dreams


# ---------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the queries of a decode step: one row of each head, where the launch counts
        dict(name="turn_token", kind="turn", dtype="bf16", batch=4, heads=32, rows=1, d=128, rot=128, pairs="half",
             base=1e4, scaling="none", factor=1.0, at="next", far=4096, gain=1.0),
        # part of the head, interleaved pairs, fp32, far positions given one by one, a context that was stretched
        dict(name="turn_part_f32", kind="turn", dtype="f32", batch=2, heads=8, rows=437, d=64, rot=32, pairs="adjacent",
             base=5e5, scaling="parts", factor=8.0, at="given", far=1000000, gain=1.2079),
        # a long prompt's queries: a copy's bandwidth
        dict(name="turn_prompt", kind="turn", dtype="bf16", batch=1, heads=28, rows=8192, d=128, rot=128, pairs="half",
             base=1e6, scaling="linear", factor=4.0, at="next", far=0, gain=1.0),
        # a LLaVA-1.6-7B layer's step of four sequences: 60 drafted nodes each
        dict(name="append_tree_7b", kind="append", dtype="bf16", batch=4, hq=32, hkv=32, d=128, rot=128, pairs="half",
             base=1e4, scaling="none", factor=1.0, at="tree", gain=1.0, lo=500, hi=800, rows=60, rlo=60, depth=6,
             branch=4, page=64, paired=False),
        # ragged prompts of a padded batch, behind cached prefixes, over few KV heads
        dict(name="append_prompt_gqa", kind="append", dtype="bf16", batch=4, hq=28, hkv=4, d=128, rot=128, pairs="half",
             base=1e6, scaling="parts", factor=4.0, at="next", gain=1.1386, lo=0, hi=700, rows=2049, rlo=300, depth=0,
             branch=1, page=32, paired=True),
        # a step of eight sequences over 8 KV heads, in 8 bits: 60 nodes in, their path compacted, the cache read back
        dict(name="store8_tree", kind="store8", dtype="bf16", batch=8, hq=32, hkv=8, d=128, rot=128, pairs="half",
             base=5e5, scaling="none", factor=1.0, at="tree", gain=1.0, lo=37, hi=130, rows=60, rlo=60, depth=6,
             branch=4, page=16, paired=False),
        # a LLaVA-1.6-7B prompt (2880 image and 256 text tokens) into 8 bits
        dict(name="store8_prompt_7b", kind="store8", dtype="bf16", batch=1, hq=32, hkv=32, d=128, rot=128, pairs="half",
             base=1e4, scaling="none", factor=1.0, at="next", gain=1.0, lo=0, hi=0, rows=3136, rlo=3136, depth=0,
             branch=1, page=64, paired=False),
        # single tokens of a few sequences, window and sinks: the launch and the latency of the reads count
        dict(name="verify8_token_sinks", kind="verify8", batch=4, hq=32, hkv=8, d=128, lo=1500, hi=8192, rows=1, rlo=1,
             depth=0, branch=1, page=16, window=1024, sinks=4, mask=False, paired=False),
        # an ordinary step at batch 1: one LLaVA-1.6-7B layer and a 60-node tree
        dict(name="verify8_7b_layer", kind="verify8", batch=1, hq=32, hkv=32, d=128, lo=3136, hi=3136, rows=60, rlo=60,
             depth=6, branch=4, page=64, window=0, sinks=0, mask=False, paired=False),
        # single tokens of long contexts: the cache is read once, at the memory's rate
        dict(name="verify8_token_long", kind="verify8", batch=8, hq=32, hkv=8, d=128, lo=16384, hi=32768, rows=1, rlo=1,
             depth=0, branch=1, page=64, window=0, sinks=0, mask=False, paired=False),
        # ragged pieces of prompts behind what is cached of them, 64 columns
        dict(name="prompt8_piece", kind="prompt8", batch=3, hq=24, hkv=8, d=64, lo=100, hi=2050, rows=333, rlo=7, depth=0,
             branch=1, page=16, window=0, sinks=0, mask=False, paired=True),
        # a long prompt over few KV heads: the largest product
        dict(name="prompt8_gqa_long", kind="prompt8", batch=1, hq=28, hkv=4, d=128, lo=0, hi=0, rows=8192, rlo=8192,
             depth=0, branch=1, page=64, window=0, sinks=0, mask=False, paired=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _tree_shape(rng, most):
    rows = 1 if rng.random() < 0.2 else _log_int(rng, 1, most)
    depth = rng.randint(min(3, rows - 1), min(8, rows - 1)) if rows > 1 else 0
    return dict(rows=rows, rlo=rows, depth=depth, branch=rng.randint(4, 6) if rows <= 60 else 6)


def _chain_shape(rng, most):
    rows = _log_int(rng, 1, most)
    return dict(rows=rows, rlo=int(rows * rng.uniform(0.0, 1.0)), depth=0, branch=1)


def _window(rng, hi):
    if rng.random() < 0.5:
        return dict(window=0, sinks=0)
    return dict(window=_log_int(rng, 1, max(2, hi)), sinks=rng.choice((0, 1, 4, 17, 64)))


def _rotation(rng, d):
    scaling = rng.choice(("none", "none", "linear", "parts"))
    return dict(d=d, rot=rng.choice((d, d, d, d // 2 // 16 * 16, 16)), pairs=rng.choice(("half", "half", "adjacent")),
                base=rng.choice((1e4, 5e5, 1e6)), scaling=scaling,
                factor=1.0 if scaling == "none" else round(math.exp(rng.uniform(0.2, 3.0)), 3),
                gain=1.0 if rng.random() < 0.7 else round(rng.uniform(1.0, 1.4), 4))


_HEADS = ((32, 32), (40, 40), (28, 4), (32, 8), (24, 8), (16, 16), (8, 2), (7, 1))
_PAGES = (16, 16, 32, 64, 128, 256)


def draw(rng):
    """One more case of the listed kinds, its sizes spread over the range that they cover."""
    kind = rng.choice(("turn", "append", "store8", "store8", "verify8", "verify8", "verify8", "prompt8", "prompt8"))
    if kind == "turn":
        heads, rows = rng.randint(1, 40), _log_int(rng, 1, 8192)
        d, dtype = rng.choice((64, 80, 96, 128, 128)), rng.choice(("bf16", "bf16", "f32"))
        most = 28 * 8192 * 128 // (2 if dtype == "f32" else 1)
        batch = max(1, min(_log_int(rng, 1, 64), most // (heads * rows * d)))
        if heads * rows * d > most:
            heads = max(1, most // (rows * d))
        at = rng.choice(("next", "given", "tree")) if rows <= 128 else rng.choice(("next", "given"))
        return dict(kind="turn", dtype=dtype, batch=batch, heads=heads, rows=rows, at=at, far=_log_int(rng, 1, 1000000),
                    **_rotation(rng, d))
    common = dict(page=rng.choice(_PAGES), paired=rng.random() < 0.3)
    hq, hkv = rng.choice(_HEADS)
    d = rng.choice((64, 128, 128))
    if kind in ("append", "store8"):
        at = rng.choice(("tree", "next"))
        shape = _tree_shape(rng, 128) if at == "tree" else _chain_shape(rng, 4096)
        hi = _log_int(rng, 1, 2048 if kind == "append" else 256) if rng.random() < 0.7 else 0
        most = 40 * 4096 * 128
        batch = max(1, min(_log_int(rng, 1, 16), most // ((hq + 2 * hkv) * d * (shape["rows"] + hi))))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        return dict(kind=kind, dtype=dtype, batch=batch, hq=hq, hkv=hkv, at=at, lo=int(hi * rng.uniform(0.0, 1.0)),
                    hi=hi, **_rotation(rng, d), **shape, **common)
    if kind == "verify8":
        hi = _log_int(rng, 1, 32768)
        shape = _tree_shape(rng, 128)
        most = 8 * 8 * 32768
        if hi > 8192 and shape["rows"] > 16:
            hi //= 4
        batch = max(1, min(_log_int(rng, 1, 16), most // (hkv * hi), int(4e9 / 128 / (hq * shape["rows"] * hi))))
        return dict(kind="verify8", batch=batch, hq=hq, hkv=hkv, d=d, lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi,
                    mask=rng.random() < 0.3, **_window(rng, hi), **shape, **common)
    hq, hkv = rng.choice(((32, 32), (28, 4), (32, 8), (24, 8), (8, 2), (7, 1)))
    shape = _chain_shape(rng, 8192)
    rows = shape["rows"]
    hi = 0 if rng.random() < 0.5 else _log_int(rng, 1, 8192)
    most = 28 * 8192 * 4096     # the longest listed prompt's scores
    if hq * rows * (hi + rows / 2) > most:
        hi = 0
    if hq * rows * rows / 2 > most:
        hq, hkv = 28, 4
    batch = max(1, min(rng.randint(1, 8), int(most / (hq * rows * (hi + rows / 2)))))
    return dict(kind="prompt8", batch=batch, hq=hq, hkv=hkv, d=d, lo=int(hi * rng.uniform(0.0, 1.0)), hi=hi, mask=False,
                **_window(rng, hi + rows), **shape, **common)


# ------------------------------------------------------------------------------------------------------- inputs
class _Inputs:
    """Seeded draws on the device (tensors) and the host (trees, lengths, tables)."""

    def __init__(self, case, seed):
        self.host = np.random.default_rng(seed)
        self.gen = torch.Generator(device=DEVICE)
        self.gen.manual_seed(int(seed))
        self.case = case
        self.dtype = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16

    def normal(self, shape, dtype=None, std=1.0):
        return torch.empty(shape, dtype=dtype or self.dtype, device=DEVICE).normal_(0.0, std, generator=self.gen)

    def keys(self, shape, dtype=None):
        """Rows as a projection makes them: some columns are large in every row, and rows differ in size."""
        x = self.normal(shape, torch.float32)
        x *= torch.exp(self.normal((shape[-1],), torch.float32, 0.7))
        x *= torch.exp(self.normal(tuple(shape[:-1]) + (1,), torch.float32, 0.3))
        return x.to(dtype or self.dtype)

    def lengths(self, lo, hi, batch):
        """Lengths lo..hi, the longest one present (a server sizes its bound by it)."""
        n = self.host.integers(lo, hi + 1, size=batch).astype(np.int32)
        n[int(self.host.integers(batch))] = hi
        return n

    def pool(self, pages):
        """(k, v) pages: two tensors, or the two halves of every page of one."""
        c = self.case
        tail = (c["hkv"], c["page"], c["d"])
        if c["paired"]:
            both = self.keys((pages, 2) + tail)
            return both[:, 0], both[:, 1]
        return self.keys((pages,) + tail), self.keys((pages,) + tail)

    def pool8(self, pages):
        """(k, v, k_scales, v_scales) in 8 bits: as _pool, the scales of a pool beside one another likewise."""
        c = self.case
        tail, flat = (c["hkv"], c["page"], c["d"]), (c["hkv"], c["page"] // 16)
        codes = torch.empty((pages, 2) + tail, dtype=torch.uint8, device=DEVICE)
        bytes_ = torch.empty((pages, 2) + flat, dtype=torch.uint8, device=DEVICE)
        step = max(1, 2 ** 28 // (c["hkv"] * c["page"] * c["d"]))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            for half in range(2):
                x = self.keys((n,) + tail, torch.float32).reshape(n, c["hkv"], -1, 16 * c["d"])
                at = _scale_byte(x.abs().amax(dim=3))
                codes[p:p + n, half] = (x * _power(254 - at)[..., None]).to(_E4M3).view(torch.uint8).reshape((n,) + tail)
                bytes_[p:p + n, half] = at.to(torch.uint8)
        if not c["paired"]:
            k, v, ks, vs = (t[:, i].contiguous() for t in (codes, bytes_) for i in range(2))
        else:
            k, v, ks, vs = (t[:, i] for t in (codes, bytes_) for i in range(2))
        return k.view(_E4M3), v.view(_E4M3), ks.view(_E8M0), vs.view(_E8M0)

    def table(self, counts, width, pages):
        """Every sequence's pages from anywhere in the pool, as after some time of service; -1 past them."""
        ids = self.host.permutation(pages).astype(np.int32)
        table = np.full((len(counts), width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(counts):
            table[b, :n] = ids[at:at + n]
            at += n
        return _device(table)

    def frequencies(self):
        return _device(_frequencies(self.case))


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


def _frequencies(case):
    """Radians a position for every pair, in 64 bits: base^(-2i/rot), slowed by `factor` in a stretched context: all of
    them, or (parts) those whose turns within the 4096 positions of training number 1 at most, and in part up to 32."""
    f = float(case["base"]) ** (-2.0 * np.arange(case["rot"] // 2, dtype=np.float64) / case["rot"])
    if case["scaling"] == "linear":
        return f / case["factor"]
    if case["scaling"] == "parts":
        keep = np.clip((4096.0 * f / (2.0 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        return f * (keep + (1.0 - keep) / case["factor"])
    return f


def _trees(r, case):
    depth, branch = case.get("depth"), case.get("branch")
    if depth is None:       # (a rotation alone: any tree)
        depth, branch = min(6, case["rows"] - 1), 6
    return np.stack([_tree(r.host, case["rows"], depth, branch) for _ in range(case["batch"])])


def _prepare_turn(case, seed):
    r = _Inputs(case, seed)
    batch, rows = case["batch"], case["rows"]
    # a projection's output: token by token, a token's heads side by side
    x = r.normal((batch, rows, case["heads"], case["d"])).transpose(1, 2)
    lens = r.lengths(0, case["far"], batch)
    s = dict(kind="turn", case=case, x=x, freq=r.frequencies(), kv_len=None, given=None, parent=None)
    if case["at"] == "given":
        s["given"] = _device(r.host.integers(0, case["far"] + 1, size=(batch, rows)).astype(np.int32))
        s["where"] = s["given"]
        return s
    s["kv_len"] = _device(lens)
    step = np.arange(rows, dtype=np.int32)[None]
    if case["at"] == "tree":
        parent = _trees(r, case)
        s["parent"], step = _device(parent), _depths(parent)
    s["where"] = _device(lens[:, None] + step)
    return s


def _prepare_rows(case, seed, pool8):
    r = _Inputs(case, seed)
    batch, rows, page = case["batch"], case["rows"], case["page"]
    lengths, live = r.lengths(case["lo"], case["hi"], batch), r.lengths(case["rlo"], rows, batch)
    counts, width = -(-(lengths + live) // page), -(-(case["hi"] + rows) // page)
    new = (batch, rows, case["hkv"], case["d"])
    s = dict(kind=case["kind"], case=case, kv_len=_device(lengths), row_len=_device(live), parent=None,
             freq=r.frequencies(), q=r.normal((batch, rows, case["hq"], case["d"])).transpose(1, 2),
             k_new=r.keys(new).transpose(1, 2), v_new=r.keys(new).transpose(1, 2),
             table=r.table(counts, width, batch * width + 1))
    step = np.broadcast_to(np.arange(rows, dtype=np.int32), (batch, rows))
    if case["at"] == "tree":
        parent = _trees(r, case)
        step = _depths(parent)
        path = np.full((batch, rows), -1, dtype=np.int32)
        taken = np.zeros(batch, dtype=np.int32)
        for b in range(batch):      # the way from the root to some node
            i = int(r.host.integers(rows))
            taken[b] = step[b, i]
            while i >= 0:
                path[b, step[b, i]] = i
                i = int(parent[b, i])
        s.update(parent=_device(parent), path=_device(path), taken=_device(taken), row_len=None)
    s["where"] = _device(lengths[:, None] + step)
    if pool8:
        s["k"], s["v"], s["ks"], s["vs"] = r.pool8(batch * width + 1)
    else:
        s["k"], s["v"] = r.pool(batch * width + 1)
    return s


def _prepare_append(case, seed):
    return _prepare_rows(case, seed, False)


def _prepare_store8(case, seed):
    return _prepare_rows(case, seed, True)


def _prepare_verify8(case, seed):
    r = _Inputs(case, seed)
    batch, rows, page = case["batch"], case["rows"], case["page"]
    lengths, parent = r.lengths(case["lo"], case["hi"], batch), _trees(r, case)
    counts, width = -(-(lengths + rows) // page), -(-(case["hi"] + rows) // page)
    see = _ancestors(parent)
    if case["mask"]:
        see &= r.host.random(see.shape) < 0.7   # a caller's own mask: some ancestors hidden, now and then all of a row
    pages = batch * width + 1
    k, v, ks, vs = r.pool8(pages)
    return dict(kind="verify8", case=case, q=r.normal((batch, case["hq"], rows, case["d"]), std=0.5), k=k, v=v, ks=ks,
                vs=vs, table=r.table(counts, width, pages), kv_len=_device(lengths), parent=_device(parent),
                see=_device(see), deep=_device(_depths(parent)), mask=_device(_mask_bits(see)) if case["mask"] else None)


def _prepare_prompt8(case, seed):
    r = _Inputs(case, seed)
    batch, rows, page = case["batch"], case["rows"], case["page"]
    lengths, live = r.lengths(case["lo"], case["hi"], batch), r.lengths(case["rlo"], rows, batch)
    # a table wide enough for the padded rows of the longest prefix, as a server sizes it
    counts, width = -(-(lengths + live) // page), -(-(case["hi"] + rows) // page)
    pages = batch * width + 1
    k, v, ks, vs = r.pool8(pages)
    return dict(kind="prompt8", case=case, q=r.normal((batch, case["hq"], rows, case["d"]), std=0.5), k=k, v=v, ks=ks,
                vs=vs, table=r.table(counts, width, pages), kv_len=_device(lengths), row_len=_device(live))


def prepare(case, seed):
    return globals()["_prepare_" + case["kind"]](case, seed)


# ------------------------------------------------------------------------------------- the framework's operators
def _own_turn(s):
    case = s["case"]
    return _dreams().rope(s["x"], s["freq"], kv_len=s["kv_len"], positions=s["given"], parent=s["parent"],
                          interleaved=case["pairs"] == "adjacent", amplitude=case["gain"])


def _own_append(s):
    case = s["case"]
    q = _dreams().paged_append_rope(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["kv_len"], s["freq"],
                                    row_len=s["row_len"], q=s["q"], parent=s["parent"],
                                    interleaved=case["pairs"] == "adjacent", amplitude=case["gain"])
    return dict(q=q, k=s["k"], v=s["v"])


def _own_store8(s):
    dreams, case = _dreams(), s["case"]
    q = dreams.paged_append_e4m3(s["k_new"], s["v_new"], s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"],
                                 row_len=s["row_len"], frequencies=s["freq"], q=s["q"], parent=s["parent"],
                                 interleaved=case["pairs"] == "adjacent", amplitude=case["gain"])
    if case["at"] == "tree":
        held = dreams.paged_kv_commit_e4m3(s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"], s["path"],
                                           s["taken"])
    else:
        held = s["kv_len"] + s["row_len"]
    k, v = dreams.paged_read_e4m3(s["k"], s["v"], s["ks"], s["vs"], s["table"], held, case["hi"] + case["rows"])
    return dict(q=q, k=k, v=v, held=held)


def _own_verify8(s):
    case = s["case"]
    return _dreams().paged_verify_attn_e4m3(s["q"], s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"],
                                            parent=s["parent"], tree_mask=s["mask"], window=case["window"],
                                            sinks=case["sinks"], max_kv_len=max(1, case["hi"]))


def _own_prompt8(s):
    case = s["case"]
    return _dreams().paged_prompt_attn_e4m3(s["q"], s["k"], s["v"], s["ks"], s["vs"], s["table"], s["kv_len"],
                                            s["row_len"], window=case["window"], sinks=case["sinks"],
                                            max_kv_len=max(1, case["hi"]))


# ------------------------------------------------------------------------------------------------ the plain forms
def _power(byte):
    """2^(byte - 127), exactly."""
    return (byte.int() << 23).view(torch.float32)


def _scale_byte(top):
    """The least e8m0 byte (1 at least) at which values up to `top` are at most 448 = 1.75 * 2^8."""
    bits = top.view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=1)


def _rotated(x, s):
    """x [B, heads, N, D] turned by the positions s["where"] [B, N], in 32 bits (the angles in 64)."""
    case, x = s["case"], x.float()
    rot = case["rot"]
    angle = s["where"].double()[:, None, :, None] * s["freq"]
    cos, sin = torch.cos(angle).float() * case["gain"], torch.sin(angle).float() * case["gain"]
    if case["pairs"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., rot:]), dim=3)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    pairs = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=4).flatten(3)
    return torch.cat((pairs, x[..., rot:]), dim=3)


def _plain_turn(s):
    return _rotated(s["x"], s).to(s["x"].dtype).contiguous()


def _live(s):
    """[B, N]: a sequence's own rows of a padded batch."""
    n = torch.arange(s["case"]["rows"], device=DEVICE)[None]
    return n < s["row_len"][:, None] if s["row_len"] is not None else (n >= 0).expand(s["case"]["batch"], -1)


def _queries(s):
    q = _rotated(s["q"], s).to(s["q"].dtype)
    return torch.where(_live(s)[:, None, :, None], q, torch.zeros_like(q)).contiguous()


def _place(s, slot):
    """(pages, rows) of slots [B, ...]; past the table: of its last entry."""
    page, table = s["case"]["page"], s["table"]
    flat = slot.reshape(slot.shape[0], -1)
    ids = table.gather(1, (flat // page).clamp(max=table.shape[1] - 1)).reshape(slot.shape)
    return ids.long(), slot % page


def _plain_append(s):
    slot = s["kv_len"].long()[:, None] + torch.arange(s["case"]["rows"], device=DEVICE)
    live = _live(s)
    ids, row = _place(s, slot)
    for pool, new in ((s["k"], _rotated(s["k_new"], s)), (s["v"], s["v_new"])):
        pool[ids[live], :, row[live]] = new.transpose(1, 2)[live].to(pool.dtype)
    return dict(q=_queries(s), k=s["k"], v=s["v"])


def _blocks(s):
    """Slots [B, blocks, 16] of every 16-slot block that a sequence's new rows can touch."""
    first = s["kv_len"].long() // 16
    count = (15 + s["case"]["rows"] + 15) // 16
    return (first[:, None] + torch.arange(count, device=DEVICE))[:, :, None] * 16 + torch.arange(16, device=DEVICE)


def _rescaled(codes, by):
    """Codes as values times 2^by (a byte, 127 + by), rounded to e4m3 again."""
    return (codes.view(_E4M3).float() * _power(by)).to(_E4M3).view(torch.uint8)


def _put8(pool, scales, ids, row, at, codes, byte, rows_too, blocks_too):
    """Codes [B, blocks, 16, heads, D] into their slots where rows_too, scales [B, blocks, heads] where blocks_too."""
    pool.view(torch.uint8)[ids[rows_too], :, row[rows_too]] = codes[rows_too]
    scales.view(torch.uint8)[ids[..., 0][blocks_too], :, at[blocks_too]] = byte[blocks_too].to(torch.uint8)


def _append8(s, pool, scales, new):
    """Rows `new` [B, heads, N, D] (32 bits) into their blocks."""
    case, length = s["case"], s["kv_len"].long()[:, None, None]
    slot = _blocks(s)
    ids, row = _place(s, slot)
    at = row[..., 0] // 16
    i = slot - length
    live = s["row_len"].long()[:, None, None] if s["row_len"] is not None else case["rows"]
    fresh, held = (i >= 0) & (i < live), i < 0
    touched = fresh.any(dim=2)
    batch = torch.arange(case["batch"], device=DEVICE)[:, None, None]
    x = new.transpose(1, 2)[batch, i.clamp(0, case["rows"] - 1)]                   # [B, blocks, 16, heads, D]
    here = fresh[..., None, None]
    top = torch.where(here, x, torch.zeros_like(x)).abs().amax(dim=(2, 4))
    old = scales.view(torch.uint8)[ids[..., 0], :, at].int()
    byte = torch.maximum(_scale_byte(top), torch.where(held.any(dim=2)[..., None], old, torch.zeros_like(old)))
    codes = torch.where(here, (x * _power(254 - byte)[:, :, None, :, None]).to(_E4M3).view(torch.uint8),
                        _rescaled(pool.view(torch.uint8)[ids, :, row],
                                  127 + (old - byte).clamp(min=-127)[:, :, None, :, None]))
    _put8(pool, scales, ids, row, at, codes, byte, (fresh | held) & touched[..., None], touched)


def _commit8(s, pool, scales):
    """The path's rows behind the committed prefix."""
    case, length = s["case"], s["kv_len"].long()[:, None, None]
    slot = _blocks(s)
    ids, row = _place(s, slot)
    at, i = row[..., 0] // 16, slot - length
    path = s["path"].long().gather(1, i.clamp(0, case["rows"] - 1).flatten(1)).reshape(i.shape)
    mine = (i >= 0) & (i <= s["taken"].long()[:, None, None])
    moved = mine & (path > i)
    stay = (i < 0) | (mine & ~moved)
    from_ids, from_row = _place(s, length + torch.where(moved, path, i.clamp(min=0)))
    from_ids, from_row = torch.where(moved, from_ids, ids), torch.where(moved, from_row, row)
    source = scales.view(torch.uint8)[from_ids, :, from_row // 16].int()           # [B, blocks, 16, heads]
    live = (moved | stay)[..., None]
    byte = torch.where(live, source, torch.zeros_like(source)).amax(dim=2)
    codes = _rescaled(pool.view(torch.uint8)[from_ids, :, from_row], 127 + (source - byte[:, :, None])[..., None])
    touched = mine.any(dim=2)
    _put8(pool, scales, ids, row, at, codes, byte, (moved | stay) & touched[..., None], touched)


def _read8(s, pool, scales, length, slots):
    """The first `slots` slots of every sequence as values [B, heads, slots, D], 0 from its length on."""
    slot = torch.arange(slots, device=DEVICE)[None].expand(s["case"]["batch"], -1)
    ids, row = _place(s, slot)
    x = pool.view(torch.uint8)[ids, :, row].view(_E4M3).float()                    # [B, slots, heads, D]
    x = x * _power(scales.view(torch.uint8)[ids, :, row // 16])[..., None]
    return torch.where((slot < length[:, None])[..., None, None], x, torch.zeros_like(x)).transpose(1, 2).contiguous()


def _plain_store8(s):
    case = s["case"]
    _append8(s, s["k"], s["ks"], _rotated(s["k_new"], s))
    _append8(s, s["v"], s["vs"], s["v_new"].float())
    if case["at"] == "tree":
        _commit8(s, s["k"], s["ks"])
        _commit8(s, s["v"], s["vs"])
        held = s["kv_len"] + s["taken"] + 1
    else:
        held = s["kv_len"] + s["row_len"]
    slots = case["hi"] + case["rows"]
    return dict(q=_queries(s), k=_read8(s, s["k"], s["ks"], held, slots).bfloat16(),
                v=_read8(s, s["v"], s["vs"], held, slots).bfloat16(), held=held)


def _attend(q, k, v, see):
    """softmax over the keys in sight: q [B, heads, rows, D], k and v [B, KV heads, keys, D], see [B, rows, keys].  A row
    that sees nothing: 0 and -inf."""
    batch, hq, rows, d = q.shape
    hkv = k.shape[1]
    z = torch.matmul((q.float() * (1.0 / math.sqrt(d))).reshape(batch, hkv, -1, d), k.transpose(2, 3).contiguous())
    z = z.reshape(batch, hq, rows, -1).masked_fill(~see[:, None], -math.inf)
    top = z.amax(dim=3, keepdim=True)
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(dim=3, keepdim=True)
    out = torch.matmul(p.reshape(batch, hkv, -1, p.shape[3]), v).reshape(batch, hq, rows, d)
    out = out / torch.where(total == 0, torch.ones_like(total), total)
    return out.to(q.dtype), (top + torch.log(total))[..., 0]


def _in_sight(where, keys, case):
    """[B, rows, keys]: position `where` [B, rows] of a row against position `keys` [B, keys] of a key."""
    if case["window"] == 0:
        return torch.ones((where.shape[0], where.shape[1], keys.shape[1]), dtype=torch.bool, device=DEVICE)
    return (where[:, :, None] - keys[:, None] < case["window"]) | (keys[:, None] < case["sinks"])


def _plain_verify8(s):
    case, rows, n = s["case"], s["case"]["rows"], s["kv_len"].long()
    slots = case["hi"] + rows
    slot = torch.arange(slots, device=DEVICE)[None].expand(case["batch"], -1)
    node = (slot - n[:, None]).clamp(0, rows - 1)
    prefix = slot < n[:, None]
    where = n[:, None] + s["deep"]
    at = torch.where(prefix, slot, where.gather(1, node))
    tree = s["see"].gather(2, node[:, None].expand(-1, rows, -1)) & (slot < n[:, None] + rows)[:, None]
    see = torch.where(prefix[:, None], torch.ones_like(tree), tree) & _in_sight(where, at, case)
    return _attend(s["q"], _read8(s, s["k"], s["ks"], n + rows, slots), _read8(s, s["v"], s["vs"], n + rows, slots), see)


def _plain_prompt8(s):
    case, rows, n, m = s["case"], s["case"]["rows"], s["kv_len"].long(), s["row_len"].long()
    slots = case["hi"] + rows
    slot = torch.arange(slots, device=DEVICE)[None].expand(case["batch"], -1)
    i = torch.arange(rows, device=DEVICE)[None]
    where = n[:, None] + i
    see = (slot[:, None] <= where[:, :, None]) & (i < m[:, None])[:, :, None] & _in_sight(where, slot, case)
    return _attend(s["q"], _read8(s, s["k"], s["ks"], n + m, slots), _read8(s, s["v"], s["vs"], n + m, slots), see)


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
    d, size = case["d"], 4 if case.get("dtype") == "f32" else 2
    if case["kind"] == "turn":
        values = case["batch"] * case["heads"] * case["rows"] * d
        return dict(bytes=2.0 * values * size, flops=3.0 * values * case["rot"] / d)
    hq, hkv, prefix = case["hq"], case["hkv"], (case["lo"] + case["hi"]) / 2
    rows = case["rows"] if case["kind"] == "verify8" else (case["rlo"] + case["rows"]) / 2
    if case["kind"] in ("append", "store8"):
        queries = case["batch"] * hq * (rows + case["rows"]) * d * size           # (rows past the live ones: zeros)
        new = case["batch"] * 2 * hkv * rows * d
        turned = 3.0 * case["batch"] * (hq + hkv) * rows * case["rot"]
        if case["kind"] == "append":
            return dict(bytes=queries + 2.0 * new * size, flops=turned)
        back = case["batch"] * 2 * hkv * d * ((case["hi"] + case["rows"]) * 2 + prefix
                                              + (case["depth"] / 2 if case["at"] == "tree" else rows))
        moved = case["batch"] * 2 * hkv * d * case["depth"] if case["at"] == "tree" else 0.0
        return dict(bytes=queries + new * (size + 1.0) + moved + back, flops=turned)
    window, sinks = case["window"], case["sinks"]
    if case["kind"] == "verify8":
        near = float(_seen(np.array([prefix]), window, sinks)[0])
        seen, keys = near * rows + rows * case["depth"] / 2, near + rows - 1
    else:
        at = _seen(prefix + np.arange(max(int(rows), 1)), window, sinks)
        seen, keys = float(at.sum()), min(prefix + rows, float(at[0]) + rows)
    heads = case["batch"] * hq
    moved = 2 * case["batch"] * hkv * keys * (d + 1 / 16) + 2 * heads * rows * d * 2 + heads * rows * 4
    return dict(bytes=moved, flops=4.0 * heads * seen * d)


# --------------------------------------------------------------------------------------- the same, in 64 bits
def _e4m3_values():
    """The values of the 256 codes of e4m3: sign, 4 bits of exponent (bias 7), 3 of fraction; all ones: no number."""
    code = np.arange(256)
    e, f = (code >> 3) & 15, code & 7
    v = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1.0 + f / 8.0) * 2.0 ** (e - 7.0))
    v[(code & 127) == 127] = np.nan
    return np.where(code >= 128, -v, v)


def _power64(e):
    """2^e in 64 bits, exactly, of whole numbers -160 .. 160."""
    return _device(2.0 ** np.arange(-160.0, 161.0))[e.long() + 160]


def _nearest_e4m3(x):
    """x (|x| <= 448) rounded to e4m3's numbers, ties to the even fraction: multiples of 2^(e - 3), 2^-9 at the least."""
    _, e = torch.frexp(x)
    step = _power64((e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _turned64(x, where, case):
    """Rows x [..., N, D] at positions `where` [N]: each pair as a complex number times e^(i angle)."""
    x, rot = x.double(), case["rot"]
    angle = torch.outer(where.double(), _device(_frequencies(case)))
    turn = torch.polar(torch.full_like(angle, float(case["gain"])), angle)
    y = x.clone()
    if case["pairs"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous()) * turn
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    return y


def _values64(s, name, b, slots):
    """Sequence b's slots [KV heads, slots, D] in 64 bits, each place looked up, each code's value in a table."""
    page, table = s["case"]["page"], s["table"].cpu().numpy()[b]
    at = np.arange(slots)
    ids, row = _device(table[at // page].astype(np.int64)), _device(at % page)
    x = _device(_e4m3_values())[s[name].view(torch.uint8)[ids, :, row].long()]      # [slots, KV heads, D]
    scale = _power64(s[name + "s"].view(torch.uint8)[ids, :, row // 16].long() - 127)
    return (x * scale[..., None]).transpose(0, 1).contiguous(), scale.t().contiguous()


def _blocked64(x, scale):
    """Rows x [heads, n, D] whose blocks of 16 slots (block 0 at `scale` [heads] at least) take their scales: (values in
    e4m3 times the scale, scales [heads, n])."""
    heads, n, d = x.shape
    blocks = -(-n // 16)
    y = torch.zeros((heads, blocks * 16, d), dtype=torch.float64, device=DEVICE)
    y[:, :n] = x
    y = y.reshape(heads, blocks, 16 * d)
    top = y.abs().amax(dim=2).cpu().numpy()
    with np.errstate(divide="ignore"):
        at = np.ceil(np.log2(top / 448.0))
    at = np.where(top > 448.0 * 2.0 ** at, at + 1, np.where(top <= 448.0 * 2.0 ** (at - 1), at - 1, at))    # (rounded logs)
    at = _device(np.maximum(np.where(top > 0, at, -126.0), -126.0))
    at[:, 0] = torch.maximum(at[:, 0], torch.frexp(scale)[1] - 1.0)
    size = _power64(at)[..., None]
    y = (_nearest_e4m3(y / size) * size).reshape(heads, blocks * 16, d)
    return y[:, :n], _power64(at).repeat_interleave(16, dim=1)[:, :n]


def _exact_store8(s):
    """Sequence by sequence: the last block's held rows and the new ones take its scale, the path's rows move on."""
    case = s["case"]
    slots = case["hi"] + case["rows"]
    shape = (case["batch"], case["hkv"], slots, case["d"])
    out = dict(q=torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE), held=None,
               k=torch.zeros(shape, dtype=torch.float64, device=DEVICE),
               v=torch.zeros(shape, dtype=torch.float64, device=DEVICE))
    for b in range(case["batch"]):
        n = int(s["kv_len"][b])
        m = case["rows"] if s["row_len"] is None else int(s["row_len"][b])
        where = s["where"][b, :m]
        out["q"][b, :, :m] = _turned64(s["q"][b, :, :m], where, case)
        for name in ("k", "v"):
            new = s[name + "_new"][b, :, :m]
            new = _turned64(new, where, case) if name == "k" else new.double()
            old, scale = _values64(s, name, b, n) if n else (out[name][b, :, :0], None)
            lead = n % 16
            least = scale[:, n - 1] if lead else torch.full((case["hkv"],), 2.0 ** -126, dtype=torch.float64, device=DEVICE)
            if m:
                rows, by = _blocked64(torch.cat((old[:, n - lead:], new), dim=1), least)
                if case["at"] == "tree":
                    a = int(s["taken"][b])
                    way = s["path"][b, :a + 1].long() + lead
                    take = torch.cat((torch.arange(lead, device=DEVICE), way))
                    rows, by = rows[:, take], by[:, take]
                    # a block's scale: the largest of its rows'
                    for i in range(0, rows.shape[1], 16):
                        size = by[:, i:i + 16].amax(dim=1)[:, None, None]
                        rows[:, i:i + 16] = _nearest_e4m3(rows[:, i:i + 16] / size) * size
            else:
                rows = old[:, n - lead:]
            out[name][b, :, :n - lead] = old[:, :n - lead]
            out[name][b, :, n - lead:n - lead + rows.shape[1]] = rows
    return out


def _softmax64(scores, values):
    """(out, lse) of one head's masked scores [rows, keys] in 64 bits."""
    lse = torch.logsumexp(scores, dim=1)
    p = torch.exp(scores - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    return p @ values, lse


def _exact_attention(s):
    """Row by row of the definition: every slot's place looked up in the table, every key's place compared with the
    row's."""
    case, q = s["case"], s["q"]
    batch, hq, rows, d = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full((batch, hq, rows), -math.inf, dtype=torch.float64, device=DEVICE)
    for b in range(batch):
        n = int(s["kv_len"][b])
        m = rows if case["kind"] == "verify8" else int(s["row_len"][b])
        if m == 0:
            continue
        if case["kind"] == "verify8":
            depth = s["deep"][b].cpu().numpy()
            row_at, key_at = n + depth, np.concatenate((np.arange(n), n + depth))
            sight = np.ones((m, n + m), dtype=bool)
            sight[:, n:] = s["see"][b].cpu().numpy()
        else:
            row_at, key_at = n + np.arange(m), np.arange(n + m)
            sight = key_at[None, :] <= row_at[:, None]
        if case["window"]:
            sight &= (key_at[None, :] < case["sinks"]) | (row_at[:, None] - key_at[None, :] < case["window"])
        hidden = _device(~sight)
        keys, values = _values64(s, "k", b, n + m)[0], _values64(s, "v", b, n + m)[0]
        for h in range(hq):
            g = h // (hq // case["hkv"])
            z = q[b, h, :m].double() @ keys[g].t().contiguous() / math.sqrt(d)
            out[b, h, :m], lse[b, h, :m] = _softmax64(z.masked_fill_(hidden, -math.inf), values[g])
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "turn":
        return torch.stack([_turned64(s["x"][b], s["where"][b], case) for b in range(case["batch"])])
    if case["kind"] == "append":
        q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        pools = dict(k=s["k"].double(), v=s["v"].double())
        table = s["table"].cpu().numpy()
        for b in range(case["batch"]):
            n = int(s["kv_len"][b])
            m = case["rows"] if s["row_len"] is None else int(s["row_len"][b])
            where = s["where"][b, :m]
            q[b, :, :m] = _turned64(s["q"][b, :, :m], where, case)
            at = n + np.arange(m)
            ids, row = _device(table[b][at // case["page"]].astype(np.int64)), _device(at % case["page"])
            pools["k"][ids, :, row] = _turned64(s["k_new"][b, :, :m], where, case).transpose(0, 1)
            pools["v"][ids, :, row] = s["v_new"][b, :, :m].double().transpose(0, 1)
        return dict(q=q, **pools)
    if case["kind"] == "store8":
        return _exact_store8(s)
    return _exact_attention(s)
