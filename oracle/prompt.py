"""Softmax attention over whole prompts in float64, and how far a float32 / 16-bit evaluation may be from it."""

import numpy as np


def attention(q, k, v, causal=True, scale=None):
    """q [nq, Hq, d], k, v [nk, Hkv, d] -> out [nq, Hq, d], lse [Hq, nq], spread [nq, Hq, d] (probability-weighted |v|),
    reach (largest scale * sum |q_c| |k_c|)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    nq, hq, d = q.shape
    nk, hkv = k.shape[0], k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, spread = np.zeros((nq, hq, d)), np.zeros((nq, hq, d))
    lse = np.full((hq, nq), -np.inf)
    reach = 0.0
    for h in range(hq):
        g = h // (hq // hkv)
        if nk == 0 or nq == 0:
            continue
        x = scale * (q[:, h] @ k[:, g].T)
        reach = max(reach, float(scale * np.max(np.abs(q[:, h]) @ np.abs(k[:, g]).T)))
        if causal:
            x = np.where(np.arange(nk)[None] <= np.arange(nq)[:, None] + nk - nq, x, -np.inf)
        m = x.max(axis=1)
        ok = np.isfinite(m)
        p = np.exp(x - np.where(ok, m, 0.0)[:, None])
        l = p.sum(axis=1)
        p = np.where(ok[:, None], p / np.where(ok, l, 1.0)[:, None], 0.0)
        out[:, h], spread[:, h] = p @ v[:, g], p @ np.abs(v[:, g])
        lse[h, ok] = m[ok] + np.log(l[ok])
    return out, lse, spread, reach


def logit_error(d, reach):
    """Bound of a probability's relative error from its logit: a float32 sum of d products (error at most (d + 4) 2^-24 of
    the sum of magnitudes, doubled for accumulators that truncate), the subtraction of the reference and the
    exponential's own 2^-22; doubled because the denominator has the same."""
    return 2 * (2 * (d + 4) * 2.0 ** -24 * reach + 2.0 ** -21)


def out_tolerance(out, spread, vmax, n_keys, d, reach, u_out, u_prob):
    """u_out: half a step of the output type; u_prob: of the type in which probabilities enter the product (fp16 has an
    absolute floor of 2^-25 of the row's reference, which is at most the row's sum)."""
    rel = logit_error(d, reach)
    return u_out * np.abs(out) * 1.01 + (u_prob + rel) * spread * 1.01 + n_keys * 2.0 ** -25 * vmax + 1e-30


def lse_tolerance(lse, d, reach):
    return logit_error(d, reach) + 2.0 ** -21 * np.maximum(1.0, np.abs(lse))
