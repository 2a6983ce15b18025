"""The 8-bit cache with a scale for each block of tokens and KV head, in numpy: append, attention with block masses,
eviction.  The quantizer's definition rounds the scale and the quotient to float32; float64 division followed by that
rounding is the same number."""

import numpy as np

from . import prompt

MOST = {"int8": 127.0, "e4m3": 448.0}


def e4m3_values():
    """The 127 non-negative finite values of the 8-bit float with 4 exponent and 3 significand bits, by code."""
    codes = np.arange(127)
    e, m = codes >> 3, codes & 7
    return np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))


def round_e4m3(y):
    """Nearest value (ties to the even code), saturating."""
    vals = e4m3_values()
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(vals, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - vals[lo], vals[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(vals[pick], y)


def quantize(x, code):
    """x [B, d] -> (values of the codes as float64, scale float32)."""
    x = np.asarray(x, np.float64)
    amax = np.abs(x).max() if np.isfinite(x).all() else np.inf
    if not np.isfinite(amax):
        return np.zeros_like(x), np.float32(1.0)
    scale = np.float32(amax / MOST[code])
    if not scale > 0:
        scale = np.float32(1.0)
    y = (x / np.float64(scale)).astype(np.float32).astype(np.float64)
    return (np.clip(np.rint(y), -127, 127) if code == "int8" else round_e4m3(y)), scale


class Cache:
    """codes[w] [n_pages, H, B, d] float64 values, scale[w] [n_pages, H] float32, tail[w] [n, H, B, d] float64."""

    def __init__(self, codes, scale, tail, table, code):
        self.codes, self.scale, self.tail, self.table, self.code = codes, scale, tail, table, code
        self.block = codes[0].shape[2]

    def page(self, s, b):
        p = int(self.table[s, b])
        return p if 0 <= p < self.codes[0].shape[0] else None

    def append(self, new, start, counts, first_rows):
        """new: (k, v) [total, H, d]; sequence s takes rows first_rows[s] .. + counts[s]."""
        b = self.block
        for s, (st, n, r0) in enumerate(zip(start, counts, first_rows)):
            if st < 0:
                continue
            for i in range(int(n)):
                pos = int(st) + i
                if pos >= self.table.shape[1] * b:
                    break
                for w in range(2):
                    self.tail[w][s, :, pos % b] = new[w][r0 + i]
                if pos % b == b - 1:
                    p = self.page(s, pos // b)
                    if p is None:
                        continue
                    for w in range(2):
                        for h in range(self.codes[w].shape[1]):
                            self.codes[w][p, h], self.scale[w][p, h] = quantize(self.tail[w][s, h], self.code)

    def rows(self, s, n):
        """Keys, values [m, H, d] of the tokens that are there, and each one's block."""
        b, out, blk = self.block, ([], []), []
        for j in range(-(-n // b)):
            cnt = min(b, n - j * b)
            if cnt == b:
                p = self.page(s, j)
                if p is None:
                    continue
                x = [self.codes[w][p] * self.scale[w][p].astype(np.float64)[:, None, None] for w in range(2)]
            else:
                x = [self.tail[w][s, :, :cnt] for w in range(2)]
            for w in range(2):
                out[w].append(x[w].transpose(1, 0, 2))
            blk += [j] * cnt
        h, d = self.codes[0].shape[1], self.codes[0].shape[3]
        return [np.concatenate(x) if x else np.zeros((0, h, d)) for x in out] + [np.array(blk, int)]

    def attend(self, q, lens, scale=None):
        """q [n, Hq, d] -> per sequence (out [Hq, d], lse [Hq], spread, reach, n_keys, vmax), masses [n, max_blocks]."""
        res, mass = [], np.zeros(self.table.shape)
        for s in range(q.shape[0]):
            k, v, blk = self.rows(s, max(0, int(lens[s])))
            out, lse, spread, reach = prompt.attention(q[s:s + 1], k, v, False, scale)
            if len(blk):
                hq, hkv, d = q.shape[1], k.shape[1], q.shape[2]
                for h in range(hq):
                    x = (d ** -0.5 if scale is None else scale) * (k[:, h // (hq // hkv)] @ np.asarray(q[s, h], np.float64))
                    np.add.at(mass[s], blk, np.exp(x - lse[h, 0]))
            res.append((out[0], lse[:, 0], spread[0], reach, len(blk), float(np.abs(v).max()) if v.size else 0.0))
        return res, mass


def evict(table, lens, scores, block, n_pages, budget, sink, recent):
    """Plain lists per sequence; -1 / 0 behind."""
    n, mb = table.shape
    out = {"block_table": np.full((n, mb), -1, np.int32), "scores": np.zeros((n, mb), np.float32), "lens": np.array(lens),
           "kept": np.full((n, mb), -1, np.int32), "freed": np.full((n, mb), -1, np.int32), "n_freed": np.zeros(n, np.int32)}
    for s in range(n):
        full = min(max(int(lens[s]), 0) // block, mb)
        gone = []
        if full > budget:
            cand = list(range(sink, full - recent))
            key = lambda b: (-(scores[s, b]) if scores[s, b] == scores[s, b] else np.inf, b)  # noqa: E731
            nan_last = lambda b: (scores[s, b] != scores[s, b], ) + key(b)  # noqa: E731
            gone = sorted(sorted(cand, key=nan_last)[budget - sink - recent:])
        keep = [b for b in range(mb) if b not in set(gone)]
        out["kept"][s, :len(keep)] = keep
        out["block_table"][s, :len(keep)] = table[s, keep]
        out["scores"][s, :len(keep)] = scores[s, keep]
        free = [table[s, b] for b in gone if 0 <= table[s, b] < n_pages]
        out["freed"][s, :len(free)] = free
        out["n_freed"][s] = len(free)
        out["lens"][s] = int(lens[s]) - len(gone) * block
    return out
