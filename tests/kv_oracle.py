"""The 8-bit token cache and 4-bit products from their definitions, in 64 bits
on the host: slot by slot, nothing shared with the library."""
from __future__ import annotations

import numpy as np

BLOCK = 64
TOP = {"e4m3": 448.0, "int8": 127.0}


def e4m3_table():
    """The value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3
    mantissa bits; 0x7f and 0xff are not-a-number."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = -x if s else x
    v[0x7f] = v[0xff] = np.nan
    return v


E4M3 = e4m3_table()


def decode(codes, fmt):
    codes = np.asarray(codes)
    return E4M3[codes.view(np.uint8)] if fmt == "e4m3" else codes.view(np.int8).astype(np.float64)


def encode_value(y, fmt):
    """The nearest code's value, ties to the even code; clamped."""
    y = np.clip(np.asarray(y, np.float64), -TOP[fmt], TOP[fmt])
    if fmt == "int8":
        return np.rint(np.where(np.isnan(y), 0.0, y))
    pos = E4M3[:0x7f]                                # ascending: the code is the rank
    a = np.abs(np.where(np.isnan(y), 0.0, y))
    hi = np.searchsorted(pos, a).clip(0, len(pos) - 1)
    lo = (hi - 1).clip(0)
    dl, dh = a - pos[lo], pos[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(y), np.nan, np.copysign(pos[pick], y))


def scale_for(a, fmt):
    e = -100
    while a > TOP[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def value_at(t):
    """(group, place) of slot t among a block's values."""
    return (t // 4) % 4, (t // 16) * 4 + t % 4


class Cache:
    """keys, values [block, head, slot, dim] (codes' values), scales, slot data."""

    def __init__(self, k, v, ks, vs, position, weight, fmt):
        self.k, self.v, self.ks, self.vs = k, v, ks, vs
        self.position, self.weight, self.fmt = position, weight, fmt

    @classmethod
    def read(cls, dev, fmt):
        """From a qlm.DeviceKvCache."""
        import torch
        host = lambda x: x.view(torch.uint8).cpu().numpy()  # noqa: E731
        k = decode(host(dev.k_codes), fmt)
        held = decode(host(dev.v_codes), fmt)
        v = np.empty_like(k)
        for t in range(BLOCK):
            g, p = value_at(t)
            v[:, :, t] = held[:, :, g, :, p]
        opt = lambda x, dt: None if x is None else x.cpu().numpy().astype(dt)  # noqa: E731
        return cls(k, v, dev.k_scale.cpu().numpy().astype(np.float64),
                   dev.v_scale.cpu().numpy().astype(np.float64),
                   opt(dev.position, np.int64), opt(dev.weight, np.float64), fmt)

    def put(self, codes, scale, blk, h, slots, x, fresh):
        fin = np.abs(x[np.isfinite(x)])
        need = scale_for(fin.max() if fin.size else 0.0, self.fmt)
        new = need if fresh else max(scale[blk, h], need)
        if not fresh and new > scale[blk, h]:
            codes[blk, h] = encode_value(codes[blk, h] * (scale[blk, h] / new), self.fmt)
        scale[blk, h] = new
        codes[blk, h, slots] = encode_value(x / new, self.fmt)

    def append(self, table, lengths, counts, k, v, first=None):
        """k, v [rows, heads, dim] in 64 bits, sequence after sequence."""
        r0 = 0
        for s, (length, n) in enumerate(zip(lengths, counts)):
            begin = length - n
            for j in range(max(begin, 0) // BLOCK, -(-length // BLOCK)):
                lo, hi = max(begin, 0, j * BLOCK), min(length, (j + 1) * BLOCK)
                if lo >= hi or not 0 <= table[s][j] < self.k.shape[0]:
                    continue
                rows, slots = r0 + np.arange(lo, hi) - begin, np.arange(lo, hi) - j * BLOCK
                blk = table[s][j]
                for h in range(self.k.shape[1]):
                    self.put(self.k, self.ks, blk, h, slots, k[rows, h], lo == j * BLOCK)
                    self.put(self.v, self.vs, blk, h, slots, v[rows, h], lo == j * BLOCK)
                    if self.position is not None:
                        p0 = 0 if first is None else first[s] - begin
                        self.position[blk, h, slots] = p0 + np.arange(lo, hi)
                    if self.weight is not None:
                        self.weight[blk, h, slots] = 0.0
            r0 += n

    def sequence(self, row, length, h):
        """keys, values, whether there, (block, slot) of the slots of one head."""
        j = np.arange(length) // BLOCK
        blk = np.asarray(row, np.int64)[j] if length else np.zeros(0, np.int64)
        ok = (blk >= 0) & (blk < self.k.shape[0])
        at = np.where(ok, blk, 0)
        o = np.arange(length) % BLOCK
        return (self.k[at, h, o] * self.ks[at, h][:, None],
                self.v[at, h, o] * self.vs[at, h][:, None], ok, at, o)

    def attend(self, table, lengths, counts, q, scale, decay=None):
        """Outputs and, beside them, the bound of their error (see bounds());
        with decay, updates the weights and returns their bound too."""
        rows, heads, d = q.shape
        kv = self.k.shape[1]
        g = heads // kv
        out, bound = np.zeros(q.shape), np.zeros(q.shape)
        wbound = None if self.weight is None else np.zeros(self.weight.shape)
        r0 = 0
        for s, (length, n) in enumerate(zip(lengths, counts)):
            for h in range(kv):
                K, V, ok, blk, o = self.sequence(table[s], length, h)
                total, werr = np.zeros(length), np.zeros(length)
                for t in range(n):
                    for e in range(h * g, (h + 1) * g):
                        seen = ok & (np.arange(length) <= length - n + t)
                        if not seen.any():
                            continue
                        x = q[r0 + t, e]
                        sc = scale * (K[seen] @ x)
                        # single-precision sums of d exact products, then the factors
                        mag = np.abs(scale) * (np.abs(K[seen]) @ np.abs(x))
                        ds = ((d + 8) * 2.0 ** -23) * mag.max()
                        p = np.exp(sc - sc.max())
                        p /= p.sum()
                        out[r0 + t, e] = p @ V[seen]
                        # p in half precision of the running maximum (2^-11, or
                        # 2^-30 of the maximum where that is less than a normal
                        # half), its sum and the scores in single
                        pe = p * (2.0 ** -11 + 2 * ds + (len(p) + 64) * 2.0 ** -22) + \
                            2.0 ** -30 * p.max() * 256
                        bound[r0 + t, e] = pe @ np.abs(V[seen])
                        total[seen] += p
                        werr[seen] += p * (2 * ds + (len(p) + 64) * 2.0 ** -22)
                if decay is not None and length:
                    old = self.weight[blk, h, o]
                    new = total if decay == 0 else decay * old + total
                    self.weight[blk[ok], h, o[ok]] = new[ok]
                    wbound[blk[ok], h, o[ok]] = (werr + np.abs(new) * (n * g + 4) * 2.0 ** -23)[ok]
            r0 += n
        return (out, bound) if decay is None else (out, bound, wbound)

    def evict(self, table, lengths, budget, recent):
        got = []
        for s, length in enumerate(lengths):
            row = np.asarray(table[s])
            used = row[:-(-length // BLOCK)]
            if length <= budget or ((used < 0) | (used >= self.k.shape[0])).any():
                got.append(length)
                continue
            got.append(budget)
            for h in range(self.k.shape[1]):
                K, V, _, blk, o = self.sequence(row, length, h)
                pos, w = self.position[blk, h, o].copy(), self.weight[blk, h, o].copy()
                safe = pos > pos.max() - recent
                key = [(not safe[i], np.isnan(w[i]), -w[i] if not np.isnan(w[i]) else 0.0, i)
                       for i in range(length)]
                keep = np.zeros(length, bool)
                keep[[x[3] for x in sorted(key)[:budget]]] = True
                holes = np.flatnonzero(~keep[:budget])
                moved = budget + np.flatnonzero(keep[budget:])
                for j in np.unique(holes // BLOCK):
                    mine = np.flatnonzero(holes // BLOCK == j)
                    at, b = holes[mine] % BLOCK, row[j]
                    self.put(self.k, self.ks, b, h, at, K[moved[mine]], False)
                    self.put(self.v, self.vs, b, h, at, V[moved[mine]], False)
                    self.position[b, h, at], self.weight[b, h, at] = pos[moved[mine]], w[moved[mine]]
        return got


def out_bound(out, bound, dtype):
    """The error of an output rounded to `dtype`: half a unit in the last place
    of the result on top of the bound, and the least subnormal's half."""
    u, tiny = (2.0 ** -8, 2.0 ** -134) if dtype == "bf16" else (2.0 ** -11, 2.0 ** -25)
    return bound + u * (np.abs(out) + bound) + tiny


def w4(x, codes, scale, zero, group):
    """Outputs and the bound of their error before rounding."""
    n, k = codes.shape
    gi = np.arange(k) // group
    z = np.full(scale.shape, 8.0) if zero is None else zero.astype(np.float64)
    w = (codes - z[:, gi]) * scale[:, gi]
    # single-precision sums of (16 + code) x and of x, then one multiply-add a group
    mag = np.abs(x) @ ((32.0 + codes + z[:, gi]) * np.abs(scale)[:, gi]).T
    return x @ w.T, mag * (group + 8 + k / group) * 2.0 ** -23
