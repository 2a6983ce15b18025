"""Rotary positions on one or several axes and the 16-bit paged cache, in numpy (float64)."""

import numpy as np


def rotate(x, pos, inv_freq, axes=None, interleaved=False, scale=1.0, inverse=False):
    """x [tokens, heads, d], pos [n_axes, tokens] whole numbers -> [tokens, heads, d], and the sum of magnitudes that enters
    every element (0 where it is copied)."""
    x, pos = np.asarray(x, np.float64), np.atleast_2d(np.asarray(pos))
    n = len(inv_freq)
    axes = [0] * n if axes is None else axes
    theta = np.stack([pos[a].astype(np.float64) * f for a, f in zip(axes, inv_freq)], axis=1)[:, None]
    c, s = scale * np.cos(theta), scale * np.sin(theta) * (-1.0 if inverse else 1.0)
    i, j = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    y, size = x.copy(), np.zeros_like(x)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = abs(scale) * (np.abs(x[..., i]) + np.abs(x[..., j]))
    return y, size


def rotate_tolerance(y, size, pos, inv_freq, u_out, smallest):
    """Bound of the error of a float32 evaluation rounded once to a type with half step u_out and smallest subnormal `smallest`.
    In units of the magnitudes that enter: the angle's fraction as float32 (half a step of at most pi 2^-25), cosine and sine
    (at most 2 units in the last place, 2^-22), their scaling and two products and a sum (4 roundings of 2^-24): below 2^-21 +
    2^-22 in all.  The product of position and frequency in 64 bits is off by two roundings, as the oracle's is by one."""
    far = float(np.max(np.abs(np.asarray(pos, np.float64)))) * float(np.max(np.abs(inv_freq))) if size.size else 0.0
    return 1.01 * u_out * np.abs(y) + (2.0 ** -21 + 2.0 ** -22 + 4 * far * 2.0 ** -53) * size * (1 + u_out) + smallest / 2


class Pages:
    """pools[w] [n_pages, H, B, d] float64 (keys, values), table [n_seqs, max_blocks]."""

    def __init__(self, pools, table):
        self.pools, self.table, self.block = pools, table, pools[0].shape[2]

    def place(self, s, t):
        """(page, row) of token t of sequence s, or None."""
        if t // self.block >= self.table.shape[1]:
            return None
        p = int(self.table[s, t // self.block])
        return (p, t % self.block) if 0 <= p < self.pools[0].shape[0] else None

    def append(self, new, start, counts, first_rows):
        """new: (k, v) [total, H, d]; sequence s takes rows first_rows[s] .. + counts[s]."""
        for s, (st, n, r0) in enumerate(zip(start, counts, first_rows)):
            for i in range(int(n) if st >= 0 else 0):
                at = self.place(s, int(st) + i)
                if at is not None:
                    for w in range(2):
                        self.pools[w][at[0], :, at[1]] = new[w][r0 + i]

    def rows(self, s, n):
        """Keys and values [m, H, d] of the first n tokens that are there, and which tokens these are."""
        there = [(t, self.place(s, t)) for t in range(n)]
        there = [(t, p) for t, p in there if p is not None]
        h, d = self.pools[0].shape[1], self.pools[0].shape[3]
        out = [np.stack([w[p, :, r] for _, (p, r) in there]) if there else np.zeros((0, h, d)) for w in self.pools]
        return out + [np.array([t for t, _ in there], int)]
