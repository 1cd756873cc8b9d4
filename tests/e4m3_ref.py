"""Plain definitions of rotary positions and of pages in 8 bits (numpy), for their tests.

Rotation tolerances.  Angles, sines and cosines are computed in 64 bits -- 2^-51 of the turns at most (two products' and one
constant's roundings), polynomials off by 2e-10 = 2^-32 -- and rounded to fp32 with the gain, half a step of 2^-24.  One product
and the sum add a half step each: |got - (a cos - b sin)| <= gain (|a| + |b|) (4 * 2^-24 + 2 pi 2^-51 turns).  bf16 adds half a
step of 2^-8 of the result."""
import numpy as np
import torch

TWO_PI = np.longdouble("6.283185307179586476925286766559")


def rotate(x, position, freq, gain, interleaved):
    """x [..., N, D] at position [..., N] (broadcast), freq [R/2] -> (rotated, |a| + |b| of every column (0: not rotated),
    turns), angles in 80 bits."""
    x = np.asarray(x, np.float64)
    R = 2 * len(freq)
    turns = np.asarray(position)[..., None].astype(np.longdouble) * freq.astype(np.longdouble) / TWO_PI
    angle = (turns - np.rint(turns)) * TWO_PI
    c, s = gain * np.cos(angle).astype(np.float64), gain * np.sin(angle).astype(np.float64)
    first = slice(0, R, 2) if interleaved else slice(0, R // 2)
    second = slice(1, R, 2) if interleaved else slice(R // 2, R)
    a, b = x[..., first], x[..., second]
    out, size, far = x.copy(), np.zeros_like(x), np.zeros_like(x)
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    for half in (first, second):
        size[..., half] = abs(gain) * (np.abs(a) + np.abs(b))
        far[..., half] = np.abs(turns).astype(np.float64)
    return out, size, far


def check_rotation(got, want, size, far, bf16, label):
    got = np.asarray(got, np.float64)
    tol = size * (4 * 2.0 ** -24 + 2 * np.pi * 2.0 ** -51 * far)
    if bf16:
        tol = np.where(size > 0, tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want), 0.0)   # (other columns: bit for bit)
    err = np.abs(got - want)
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (label, worst, got[worst], want[worst], tol[worst])


def values():
    """What the 256 codes stand for."""
    v = np.zeros(256)
    for code in range(256):
        e, f = (code >> 3) & 15, code & 7
        x = (1 + f / 8) * 2.0 ** (e - 7) if e else f / 8 * 2.0 ** -6
        v[code] = np.nan if code & 127 == 127 else -x if code & 128 else x
    return v


VALUES = values()


def encode(x):
    """The nearest code of every x (|x| <= 448; NaN and infinities: 0x7f, the sign aside), ties to the even code."""
    x = np.asarray(x, np.float64)
    mid = (VALUES[:126] + VALUES[1:127]) / 2
    a = np.abs(x)
    code = np.searchsorted(mid, a, side="right")          # ties up ...
    tie = np.isin(a, mid) & (code % 2 == 1)
    code = np.where(tie, code - 1, code)                    # ... unless the lower code is the even one
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_byte(top):
    """The least byte s >= 1 with top <= 448 * 2^(s - 127)."""
    s = 1
    while top > 448 * 2.0 ** (s - 127):
        s += 1
    return s


def power(byte):
    return 2.0 ** (np.asarray(byte, np.float64) - 127)


class Pool8:
    """A pool of 8 bits on the host, kept by the definition, and on the device.  codes [2, NL, P, H, ps, D] and scales
    [2, NL, P, H, ps/16] (K, V); slots that nothing was written to hold any codes, NaN among them, under any scales."""

    def __init__(self, rng, dev, NL, P, H, ps, D, paired=False):
        self.ps = ps
        self.codes = rng.integers(0, 256, size=(2, NL, P, H, ps, D)).astype(np.uint8)
        self.scales = rng.integers(100, 150, size=(2, NL, P, H, ps // 16)).astype(np.uint8)
        put = lambda x: [torch.from_numpy(np.ascontiguousarray(x[i])).to(dev) for i in range(2)]
        c, s = put(self.codes), put(self.scales)
        if paired:
            both, sboth = torch.stack(c, dim=2).contiguous(), torch.stack(s, dim=2).contiguous()
            c, s = [both[:, :, i] for i in range(2)], [sboth[:, :, i] for i in range(2)]
        self.k, self.v = (x.view(torch.float8_e4m3fn) for x in c)
        self.ks, self.vs = (x.view(torch.float8_e8m0fnu) for x in s)

    def at(self, table, slot):
        page = table[slot // self.ps]
        return page, slot % self.ps

    def append(self, half, layer, head, table, L, rows):
        """rows [n, D] (64 bits) from slot L on, block by block."""
        n = len(rows)
        for slot0 in range(L - L % 16, L + n, 16):
            if slot0 // self.ps >= len(table) or not 0 <= table[slot0 // self.ps] < self.codes.shape[2]:
                continue
            page, r0 = self.at(table, slot0)
            new = [r for r in range(16) if L <= slot0 + r < L + n]
            if not new:
                continue
            held = [r for r in range(16) if slot0 + r < L]
            top = np.abs(rows[[slot0 + r - L for r in new]])
            byte = scale_byte(np.where(np.isfinite(top), top, 0).max())
            old = int(self.scales[half, layer, page, head, r0 // 16])
            if held:
                byte = max(byte, old)
            block = self.codes[half, layer, page, head, r0:r0 + 16]
            for r in held:
                block[r] = self.moved(block[r], old, byte)
            for r in new:
                block[r] = encode(rows[slot0 + r - L] / power(byte))
            self.scales[half, layer, page, head, r0 // 16] = byte

    @staticmethod
    def moved(codes, old, byte):
        return codes if old == byte else encode(VALUES[codes] * 2.0 ** (old - byte))

    def commit(self, half, layer, head, table, L, path, A):
        P = self.codes.shape[2]
        before, sbefore = self.codes[half, layer, :, head].copy(), self.scales[half, layer, :, head].copy()
        inside = lambda slot: slot // self.ps < len(table) and 0 <= table[slot // self.ps] < P
        for slot0 in range(L - L % 16, L + A + 1, 16):
            if not inside(slot0):
                continue
            page, r0 = self.at(table, slot0)
            rows = {}
            for r in range(16):
                k = slot0 + r - L
                if k > A:
                    continue
                source = slot0 + r
                if k >= 0 and path[k] > k and inside(L + path[k]):
                    source = L + path[k]
                sp, sr = self.at(table, source)
                rows[r] = (before[sp, sr], int(sbefore[sp, sr // 16]), source != slot0 + r)
            if not any(m for _, _, m in rows.values()):
                continue
            byte = max(s for _, s, _ in rows.values())
            for r, (codes, s, _) in rows.items():
                self.codes[half, layer, page, head, r0 + r] = self.moved(codes, s, byte)
            self.scales[half, layer, page, head, r0 // 16] = byte

    def slots(self, half, layer, table, n):
        """The first n slots as values [H, n, D]."""
        H, D = self.codes.shape[3], self.codes.shape[5]
        x = np.zeros((H, n, D))
        for j in range(n):
            page, r = self.at(table, j)
            x[:, j] = VALUES[self.codes[half, layer, page, :, r]] * power(self.scales[half, layer, page, :, r // 16])[:, None]
        return x

    def same(self, live=None, label=""):
        """The device's codes and scales against the host's: all of them, or where `live` [P, ps] is set (and the scales of
        blocks with such a slot).  (Two codes of NaN are alike.)"""
        for half, (c, s) in enumerate(((self.k, self.ks), (self.v, self.vs))):
            got, gs = c.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy()
            want, ws = self.codes[half], self.scales[half]
            ok = (got == want) | (np.isnan(VALUES[got]) & np.isnan(VALUES[want]))
            oks = gs == ws
            if live is not None:
                ok |= ~live[None, :, None, :, None]
                oks |= ~live.reshape(live.shape[0], -1, 16).any(2)[None, :, None]
            assert oks.all(), (label, "KV"[half], "scales", np.argwhere(~oks)[:3], gs[~oks][:3], ws[~oks][:3])
            assert ok.all(), (label, "KV"[half], "codes", np.argwhere(~ok)[:3], got[~ok][:3], want[~ok][:3])


def spread_rows(rng, shape, dev, bf16):
    """Rows whose sizes differ by powers of ten, some columns large, a few zeros; (device, 64 bits)."""
    x = rng.standard_normal(shape) * np.exp(1.5 * rng.standard_normal(shape[:-1] + (1,))) * np.exp(
        0.7 * rng.standard_normal(shape[-1:]))
    x[rng.random(shape) < 0.02] = 0
    t = torch.from_numpy(x).to(torch.bfloat16 if bf16 else torch.float32).to(dev)
    return t, t.double().cpu().numpy()


class Cache8:
    """One layer's pool in 8 bits with every sequence's pages at random places, as paged_ref.Cache: k and v are the values in 64
    bits.  Slots that no sequence fills hold NaN and the largest codes, blocks without a filled slot any scale byte."""

    def __init__(self, rng, dev, fill, Hkv, ps, D, paired=False, width=None, spare=3, scale=1.0):
        fill = np.asarray(fill)
        B = len(fill)
        counts = -(-fill // ps)
        self.width = max(int(counts.max()), 1) if width is None else width
        P = int(counts.sum()) + spare
        ids = rng.permutation(P)
        self.table = rng.choice(np.array([-1, P, 2 ** 31 - 1, -2 ** 31], np.int64), size=(B, self.width)).astype(np.int32)
        codes = rng.choice(np.array([0x7f, 0xff, 0x7e, 0xfe], np.uint8), size=(2, P, Hkv, ps, D))
        scales = rng.integers(0, 256, size=(2, P, Hkv, ps // 16)).astype(np.uint8)
        at = 0
        for b in range(B):
            self.table[b, :counts[b]] = ids[at:at + counts[b]]
            at += counts[b]
            for j0 in range(0, fill[b], 16):
                page, r0, n = self.table[b, j0 // ps], j0 % ps, min(16, fill[b] - j0)
                for half in range(2):
                    for g in range(Hkv):
                        x = (scale if half == 0 else 1.0) * rng.standard_normal((n, D)) * 2.0 ** rng.integers(-2, 2)
                        byte = scale_byte(np.abs(x).max())
                        codes[half, page, g, r0:r0 + n] = encode(x / power(byte))
                        scales[half, page, g, r0 // 16] = byte
        values = VALUES[codes] * np.repeat(power(scales), 16, axis=3)[..., None]
        self.k, self.v = values
        c, s = (torch.from_numpy(x).to(dev) for x in (codes, scales))
        if paired:
            c, s = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c, s))
        self.kd, self.vd = (c[i].view(torch.float8_e4m3fn) for i in range(2))
        self.ksd, self.vsd = (s[i].view(torch.float8_e8m0fnu) for i in range(2))
        self.tabled = torch.from_numpy(self.table).to(dev)
        self.pages = (self.kd, self.vd, self.ksd, self.vsd, self.tabled)
