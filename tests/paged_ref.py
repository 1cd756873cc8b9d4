"""Plain 64-bit definitions of the paged cache's operators (numpy), and inputs for their tests.

Attention tolerances.  Let A[d] = sum_j p_j |v_j[d]| of a row, n its keys, and ds = (D + 4) 2^-24 scale max_j sum_d |q_d k_jd|
the error of an fp32 score (products of bf16 values are exact in fp32; D sums, the scale and the reference add one rounding
each), in the exponent a relative error of a probability.  Sums of n terms in fp32 in any order add n 2^-24, the
exponential, the division and the merges a few 2^-24 more (16 here).  fp32: |out - ref| <= A (2 ds + (n + 16) 2^-24).  bf16
adds half steps of 2^-8 (torch.finfo(bfloat16).eps / 2): the probabilities' rounding before the value product (A) and the
result's (|ref|).  lse: ds + (n + 16) 2^-24 + |lse| 2^-22."""
import numpy as np
import torch

from paper_2606_00535_amd import workload as W

NEG = -np.inf


def tree(rng, B, T, depth=6, branch=4):
    return np.stack([W.random_tree(rng, T, min(depth, T - 1), branch if T <= 60 else 6) if T > 1
                     else np.array([-1], np.int32) for _ in range(B)]).astype(np.int32)


def depths(par):
    d = np.zeros(par.shape, np.int64)
    for b in range(par.shape[0]):
        for i in range(par.shape[1]):
            j = i
            while 0 <= par[b, j] < j:
                j = par[b, j]
                d[b, i] += 1
    return d


def ancestors(par):
    B, T = par.shape
    see = np.zeros((B, T, T), bool)
    for b in range(B):
        for i in range(T):
            j = i
            see[b, i, j] = True
            while 0 <= par[b, j] < j:
                j = par[b, j]
                see[b, i, j] = True
    return see


def mask_bits(see):
    B, T, _ = see.shape
    words = (T + 63) // 64
    bits = np.zeros((B, T, words * 64), np.uint8)
    bits[:, :, :T] = see
    return np.packbits(bits, axis=2, bitorder="little").view(np.int64).reshape(B, T, words)


def sight(row_at, key_at, window, sinks):
    if window == 0:
        return np.ones((len(row_at), len(key_at)), bool)
    return (row_at[:, None] - key_at[None, :] < window) | (key_at[None, :] < sinks)


def attend(q, k, v, see, scale):
    """q [Hq, R, D], k/v [Hkv, n, D] in 64 bits, see [R, n] -> out, lse, and the tolerances' A, ds, n."""
    Hq, R, D = q.shape
    G = Hq // k.shape[0]
    out, lse = np.zeros((Hq, R, D)), np.full((Hq, R), NEG)
    size, ds, count = np.zeros((Hq, R, D)), np.zeros((Hq, R)), np.broadcast_to(see.sum(1), (Hq, R))
    if k.shape[1] == 0:
        return out, lse, size, ds, count
    for h in range(Hq):
        kk, vv = k[h // G], v[h // G]
        kk, vv = np.where(see.any(0)[:, None], kk, 0), np.where(see.any(0)[:, None], vv, 0)   # (garbage that no row sees)
        z = np.where(see, scale * (q[h] @ kk.T), NEG)
        live = see.any(1)
        m = np.where(live, z.max(1, initial=NEG), 0.0)
        p = np.where(see, np.exp(z - m[:, None]), 0.0)
        s = p.sum(1)
        w = p / np.where(live, s, 1.0)[:, None]
        out[h], size[h] = w @ vv, w @ np.abs(vv)
        with np.errstate(divide="ignore"):
            lse[h] = np.where(live, m + np.log(s), NEG)
        ds[h] = np.where(see, abs(scale) * (np.abs(q[h]) @ np.abs(kk).T), 0).max(1) * (D + 4) * 2.0 ** -24
    return out, lse, size, ds, count


def slots_of(pool, table, n):
    """The first n slots of a sequence: [Hkv, n, D]."""
    ps = pool.shape[2]
    return np.stack([pool[table[j // ps], :, j % ps] for j in range(n)], axis=1) if n else \
        np.zeros((pool.shape[1], 0, pool.shape[3]))


def verify(q, kp, vp, table, kv_len, par, see, window, sinks, scale):
    """Tree rows; see [B, T, T] which nodes a node may see."""
    B, Hq, T, D = q.shape
    dep, res = depths(par), []
    for b in range(B):
        L = int(kv_len[b])
        row_at = L + dep[b]
        key_at = np.concatenate((np.arange(L), row_at))
        vis = np.concatenate((np.ones((T, L), bool), see[b]), axis=1) & sight(row_at, key_at, window, sinks)
        res.append(attend(q[b], slots_of(kp, table[b], L + T), slots_of(vp, table[b], L + T), vis, scale))
    return [np.stack(x) for x in zip(*res)]


def prompt(q, kp, vp, table, kv_len, row_len, window, sinks, scale):
    B, Hq, N, D = q.shape
    res = []
    for b in range(B):
        L, n = int(kv_len[b]), int(row_len[b])
        at = L + np.arange(N)
        vis = (np.arange(L + n)[None, :] <= at[:, None]) & sight(at, np.arange(L + n), window, sinks)
        vis[n:] = False
        res.append(attend(q[b], slots_of(kp, table[b], L + n), slots_of(vp, table[b], L + n), vis, scale))
    return [np.stack(x) for x in zip(*res)]


def check(out, lse, ref, bf16, label):
    want, wlse, size, ds, n = ref
    got, glse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    assert np.isfinite(got).all(), label
    sums = 2 * ds + (n + 16) * 2.0 ** -24
    tol = size * sums[..., None]
    if bf16:
        tol = tol * (1 + 2.0 ** -7) + 2.0 ** -8 * (size + np.abs(want)) * (1 + 2.0 ** -7)
    err = np.abs(got - want)
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol + 1e-30).all(), (label, "out", worst, got[worst], want[worst], tol[worst])
    if glse is not None:
        empty = np.isneginf(wlse)
        assert np.array_equal(np.isneginf(glse), empty), (label, "empty rows")
        e = np.abs(np.where(empty, 0, glse) - np.where(empty, 0, wlse))
        t = ds + (n + 16) * 2.0 ** -24 + np.abs(np.where(empty, 0, wlse)) * 2.0 ** -22
        assert (e <= t).all(), (label, "lse", float((e - t).max()))
    return float(err.max())


# ---------------------------------------------------------------------------------------------------------- inputs
class Cache:
    """One layer's pool on the device with every sequence's pages at random places.  Slots that no sequence fills hold
    NaN and infinities, unused table entries numbers outside the pool."""

    def __init__(self, rng, dev, fill, Hkv, ps, D, bf16, paired=False, width=None, spare=3, scale=1.0):
        fill = np.asarray(fill)
        B = len(fill)
        counts = -(-fill // ps)
        self.width = max(int(counts.max()), 1) if width is None else width
        P = int(counts.sum()) + spare
        ids = rng.permutation(P)
        self.table = rng.choice(np.array([-1, P, 2 ** 31 - 1, -2 ** 31], np.int64), size=(B, self.width)).astype(np.int32)
        shape = (P, Hkv, ps, D)
        self.k, self.v = (rng.choice(np.array([np.nan, np.inf, -np.inf, 3e38]), size=shape) for _ in range(2))
        at = 0
        for b in range(B):
            self.table[b, :counts[b]] = ids[at:at + counts[b]]
            at += counts[b]
            for j in range(fill[b]):
                page = self.table[b, j // ps]
                self.k[page, :, j % ps] = scale * rng.standard_normal((Hkv, D))
                self.v[page, :, j % ps] = rng.standard_normal((Hkv, D))
        dt = torch.bfloat16 if bf16 else torch.float32
        both = torch.empty((P, 2) + shape[1:], dtype=dt, device=dev)
        kd, vd = (torch.from_numpy(x).to(dt).to(dev) for x in (self.k, self.v))
        self.k, self.v = kd.double().cpu().numpy(), vd.double().cpu().numpy()   # as rounded
        if paired:
            both[:, 0], both[:, 1] = kd, vd
            kd, vd = both[:, 0], both[:, 1]
        self.kd, self.vd, self.tabled = kd, vd, torch.from_numpy(self.table).to(dev)


def rounded(rng, shape, bf16, dev, std=1.0):
    x = torch.from_numpy(std * rng.standard_normal(shape)).to(torch.bfloat16 if bf16 else torch.float32).to(dev)
    return x, x.double().cpu().numpy()


def ints(x, dev):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)


# ------------------------------------------------------------------------------------------------- tables, in Python
class Tables:
    """The pages of sequences, kept by the definition: one thing after another."""

    def __init__(self, B, width, P, ps):
        self.table = np.full((B, width), -1, np.int32)
        self.count, self.kv_len = np.zeros(B, np.int32), np.zeros(B, np.int32)
        self.ref, self.ps = np.zeros(P, np.int32), ps

    def copy(self):
        t = Tables(1, 1, 1, self.ps)
        t.table, t.count, t.kv_len, t.ref = (x.copy() for x in (self.table, self.count, self.kv_len, self.ref))
        return t

    def free(self):
        return [int(p) for p in np.flatnonzero(self.ref == 0)]

    def reserve(self, want):
        granted = []
        for b in range(len(self.count)):
            hold = max(0, -(-int(want[b]) // self.ps))
            lack = max(0, hold - int(self.count[b]))
            free = self.free()
            ok = hold <= self.table.shape[1] and lack <= len(free)
            if ok:
                for p in free[:lack]:
                    self.table[b, self.count[b]] = p
                    self.ref[p] = 1
                    self.count[b] += 1
            granted.append(int(ok))
        return granted

    def fork(self, src, dst):
        """granted and the (source page, copy, rows) to copy."""
        before, granted, copies, B = self.copy(), [], [], len(self.count)
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = 0 <= s < B and 0 <= d < B and s != d and d not in dst[:i] and before.count[d] == 0
            if ok:
                n = int(before.kv_len[s])
                ok = n >= 0 and -(-n // self.ps) <= before.count[s]
            free = [p for p in self.free() if before.ref[p] == 0]
            if ok and n % self.ps and not free:
                ok = False
            granted.append(int(ok))
            if not ok:
                continue
            whole = n // self.ps
            self.table[d, :whole] = before.table[s, :whole]
            for p in before.table[s, :whole]:
                self.ref[p] += 1
            self.count[d], self.kv_len[d] = whole, n
            if n % self.ps:
                self.table[d, whole] = free[0]
                self.ref[free[0]] = 1
                self.count[d] += 1
                copies.append((int(before.table[s, whole]), free[0], n % self.ps))
        return granted, copies

    def release(self, seqs, trim=False):
        for b in dict.fromkeys(int(x) for x in seqs):
            if not 0 <= b < len(self.count):
                continue
            keep = -(-int(self.kv_len[b]) // self.ps) if trim else 0
            for c in range(keep, self.count[b]):
                self.ref[self.table[b, c]] -= 1
                self.table[b, c] = -1
            self.count[b] = min(self.count[b], keep)
            if not trim:
                self.kv_len[b] = 0

    def on(self, dev):
        return [torch.from_numpy(x.copy()).to(dev) for x in (self.table, self.count, self.kv_len, self.ref)]

    def same(self, tensors):
        for x, t, name in zip((self.table, self.count, self.kv_len, self.ref), tensors, ("table", "count", "kv_len", "ref")):
            got = t.cpu().numpy()
            assert np.array_equal(got, x), (name, got, x)
