"""Softmax attention over whole prompts in float64, and how far a float32 / 16-bit evaluation may be from it."""

import numpy as np


def _visible(nq, nk, places, n_tokens):
    """Key j is token places[j] of n_tokens, the queries are the last nq of them."""
    places = np.arange(nk) if places is None else np.asarray(places)
    return places[None] <= np.arange(nq)[:, None] + (nk if n_tokens is None else n_tokens) - nq


def attention(q, k, v, causal=True, scale=None, places=None, n_tokens=None):
    """q [nq, Hq, d], k, v [nk, Hkv, d] -> out [nq, Hq, d], lse [Hq, nq], spread [nq, Hq, d] (probability-weighted |v|),
    reach (largest scale * sum |q_c| |k_c|).  places, n_tokens: the keys are these tokens of n_tokens (default: all)."""
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
            x = np.where(_visible(nq, nk, places, n_tokens), x, -np.inf)
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
    """u_out: half a step of the output type; u_prob: of the type in which probabilities enter the product.  fp16 has an absolute
    floor of 2^-25 of the row's reference, which is at most the row's sum, where the reference is the largest logit (the kernels
    for 16-bit keys set it 2^7 lower and are within 2^-32).  bf16 has the range of float32 and no such floor: what is left is the
    float32 sum of n_keys products, a rounding of 2^-24 of the sum of magnitudes for each."""
    rel = logit_error(d, reach)
    rest = n_keys * (2.0 ** -25 * vmax if u_prob < 2.0 ** -9 else 2.0 ** -24 * spread)
    return u_out * np.abs(out) * 1.01 + (u_prob + rel) * spread * 1.01 + rest + 1e-30


def lse_tolerance(lse, d, reach):
    return logit_error(d, reach) + 2.0 ** -21 * np.maximum(1.0, np.abs(lse))


def roundings(q, k, v, causal=True, scale=None):
    """What independent roundings of the probabilities add up to: sum_j p_j^2 v_j^2 [nq, Hq, d], the largest probability of a row
    [nq, Hq], sum_j v_j^2 over the keys [Hq, d]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    nq, hq, d = q.shape
    nk, hkv = k.shape[0], k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    s2, top, v2 = np.zeros((nq, hq, d)), np.zeros((nq, hq)), np.zeros((hq, d))
    for h in range(hq):
        g = h // (hq // hkv)
        x = scale * (q[:, h] @ k[:, g].T)
        if causal:
            x = np.where(np.arange(nk)[None] <= np.arange(nq)[:, None] + nk - nq, x, -np.inf)
        p = np.exp(x - x.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        s2[:, h], top[:, h], v2[h] = (p * p) @ (v[:, g] ** 2), p.max(axis=1), (v[:, g] ** 2).sum(axis=0)
    return s2, top, v2


def rms_tolerance(out, s2, top, v2, d, reach, u_out, u_prob, subnormal):
    """Bound of the root mean square of an output's error over many elements, for values that are drawn independently of queries
    and keys with mean zero.  A rounding to nearest is off by at most half a step u and has a mean square of at most u^2, and
    those of different keys and elements are independent of each other, so that their squares add up; a probability that fp16
    holds as a subnormal (`subnormal`) is off by at most 2^-25 of the row's reference, which is at most its largest probability.
    The logits' errors depend on queries and keys alone: weighted with the values their squares add up too, and in the
    denominator they move a row by at most their bound."""
    rel = logit_error(d, reach)
    low = (2.0 ** -25 * top[..., None]) ** 2 * v2[None] if subnormal else 0.0
    return np.sqrt(np.mean(((u_out + rel) * out) ** 2 + (u_prob ** 2 + rel ** 2) * s2 + low)) + 1e-30
