"""The 16-bit paged cache (append with rotary positions, attention of a chunk of new tokens) and the rotation by itself: cases,
plain forms, exact forms.

Shapes are those of the decode workloads of this library (Llama-3-8B: 32 / 8 heads of 128; Qwen2.5-7B: 28 / 4 heads of
128; the tiny test shapes with heads of 64) and their contexts (2k to 64k), window sizes 16 to 128 as page sizes.

Every case is one call; `op` says which:

  rope    queries and keys rotated to their positions, which have one axis (text) or three (time, height, width); `rot` of the
          `d` channels are rotated; inverse: the transposed rotation, which is the gradient.
  append  new tokens into the paged cache, keys rotated on the way, queries rotated beside them.
  attn    the new tokens of every sequence, in the cache already, attend over its pages, causally.  `max_q` new tokens at most,
          behind up to `prefix` cached ones; mixed: the first sequence has `max_q`, every other one has one.
"""

import math
import random

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_HEADS = [(32, 8, 128), (28, 4, 128), (8, 8, 64), (4, 2, 64), (16, 1, 128)]
_FAR = 131072  # positions that contexts of this library reach


# ---- cases ----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the queries and keys of one decode step of 16 users
        dict(name="rope-tokens", op="rope", hq=32, hkv=8, d=128, rot=128, axes=1, interleaved=0, base=500000, inverse=0, dtype="bf16", tokens=16),
        # a prompt of text and images in one piece: three axes
        dict(name="rope-images", op="rope", hq=28, hkv=4, d=128, rot=128, axes=3, interleaved=0, base=1000000, inverse=0, dtype="fp16", tokens=16384),
        # the gradient of a ragged batch on a small model, neighbouring channels paired, half of them rotated
        dict(name="rope-gradient", op="rope", hq=8, hkv=8, d=64, rot=32, axes=1, interleaved=1, base=10000, inverse=1, dtype="bf16", tokens=5003),
        # one token for each of 16 sequences
        dict(name="append-tokens", op="append", hq=32, hkv=8, d=128, rot=128, axes=1, interleaved=0, base=500000, dtype="bf16", block=64, n_seqs=16, max_start=8192, max_new=1),
        # four prompts at once into an empty cache
        dict(name="append-prompts", op="append", hq=32, hkv=8, d=128, rot=128, axes=1, interleaved=0, base=500000, dtype="bf16", block=64, n_seqs=4, max_start=0, max_new=16001),
        # the next piece of 12 prompts with images, small pages
        dict(name="append-pieces", op="append", hq=28, hkv=4, d=128, rot=128, axes=3, interleaved=0, base=1000000, dtype="fp16", block=16, n_seqs=12, max_start=8192, max_new=2048),
        # one user, short context, one token: the smallest step
        dict(name="attn-token", op="attn", hq=32, hkv=8, d=128, dtype="bf16", block=64, n_seqs=1, max_q=1, prefix=2047, ragged=0, mixed=0),
        # drafts of up to 5 tokens to verify, for 16 users with ragged contexts
        dict(name="attn-drafts", op="attn", hq=32, hkv=8, d=128, dtype="bf16", block=64, n_seqs=16, max_q=5, prefix=32763, ragged=1, mixed=0),
        # a token for each of 8 long documents, small pages
        dict(name="attn-64k", op="attn", hq=28, hkv=4, d=128, dtype="fp16", block=16, n_seqs=8, max_q=1, prefix=65535, ragged=0, mixed=0),
        # the next pieces of four prompts
        dict(name="attn-pieces", op="attn", hq=32, hkv=8, d=128, dtype="bf16", block=64, n_seqs=4, max_q=701, prefix=24000, ragged=1, mixed=0),
        # a server's step: a piece of one prompt between the tokens of 31 other users
        dict(name="attn-mixed", op="attn", hq=28, hkv=4, d=128, dtype="fp16", block=32, n_seqs=32, max_q=2048, prefix=16384, ragged=1, mixed=1),
        # the last piece of a document of 64k tokens
        dict(name="attn-long", op="attn", hq=32, hkv=8, d=128, dtype="bf16", block=128, n_seqs=1, max_q=8192, prefix=57344, ragged=0, mixed=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _draw_rotation(rng, d):
    return dict(rot=rng.choice([d, d, d, d // 2]), axes=rng.choice([1, 1, 3]), interleaved=int(rng.random() < 0.3), base=rng.choice([10000, 500000, 1000000]))


def draw(rng):
    op = rng.choice(["rope", "append", "attn", "attn"])
    hq, hkv, d = rng.choice(_HEADS)
    dtype, block = rng.choice(["bf16", "fp16"]), rng.choice([16, 32, 64, 128])
    if op == "rope":
        return dict(op=op, hq=hq, hkv=hkv, d=d, dtype=dtype, tokens=_log(rng, 1, 32768), inverse=int(rng.random() < 0.3), **_draw_rotation(rng, d))
    if op == "append":
        max_new = 1 if rng.random() < 0.4 else _log(rng, 2, 16384)
        n = max(1, min(_log(rng, 1, 64), 65536 // max_new))
        return dict(op=op, hq=hq, hkv=hkv, d=d, dtype=dtype, block=block, n_seqs=n, max_start=rng.choice([0, _log(rng, 1, 131072 // n)]), max_new=max_new, pick=rng.randrange(1 << 30), **_draw_rotation(rng, d))
    max_q = rng.choice([1, _log(rng, 2, 16), _log(rng, 17, 8192)])
    prefix = rng.choice([0, _log(rng, 1, 57344), _log(rng, 1024, 57344)])
    most = min(524288 // (max_q + prefix), int(5.0e8 / (max_q * (max_q + prefix))))
    n = max(1, min(_log(rng, 1, 64), most))
    return dict(op=op, hq=hq, hkv=hkv, d=d, dtype=dtype, block=block, n_seqs=n, max_q=max_q, prefix=prefix, ragged=int(rng.random() < 0.7), mixed=int(rng.random() < 0.2), pick=rng.randrange(1 << 30))


def _lens(case, longest, least=1, salt=0):
    """Lengths of the sequences: the first is the longest; the others are spread below it where the case is ragged."""
    rng = random.Random(case.get("pick", 7) + salt)
    return [longest] + [rng.randint(min(least, longest), longest) if case.get("ragged", 1) else longest for _ in range(case["n_seqs"] - 1)]


def _attn_lens(case):
    nq = [case["max_q"]] + [1] * (case["n_seqs"] - 1) if case["mixed"] else _lens(case, case["max_q"])
    return nq, [a + b for a, b in zip(nq, _lens(case, case["prefix"], 0, 1))]


def _append_lens(case):
    return _lens(case, case["max_start"], 0), _lens(case, case["max_new"], 1, 1)


def _cu(lens):
    return torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")


def _axes_of_pairs(case):
    """The axis of every pair: a quarter of them for the time, the others for height and width in halves."""
    n = case["rot"] // 2
    if case["axes"] == 1:
        return [0] * n
    t, h = n // 4, (n - n // 4) // 2
    return [0] * t + [1] * h + [2] * (n - t - h)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _rows(g, n, heads, d, dt, gain=1.0):
    return torch.randn((n, heads, d), generator=g, device="cuda").mul_(gain).to(dt)


def _positions(g, tokens, axes):
    """Text: consecutive positions from a far one on.  Images: frames of 16 x 16 patches, each a step later."""
    first = torch.randint(0, _FAR - tokens, (axes, 1), generator=g, device="cuda")
    i = torch.arange(tokens, device="cuda")
    steps = i[None] if axes == 1 else torch.stack([i // 256, i % 256 // 16, i % 16])
    return (first + steps).to(torch.int32)


def _pages(g, case, lens, filled):
    """Pools with room for every sequence, pages handed out in a shuffled order."""
    dt, b, n, hkv, d = _DT[case["dtype"]], case["block"], case["n_seqs"], case["hkv"], case["d"]
    per = torch.tensor([max(1, -(-x // b)) for x in lens], device="cuda")
    mb = int(per.max())
    n_pages = int(per.sum()) + 3
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    column = torch.arange(mb, device="cuda")[None]
    used = column < per[:, None]
    table = torch.full((n, mb), -1, dtype=torch.int32, device="cuda")
    table[used] = perm[(column + (per.cumsum(0) - per)[:, None])[used]]
    make = torch.randn if filled else torch.zeros
    args = dict(dtype=dt, device="cuda", **({"generator": g} if filled else {}))
    return {"block": b, "block_table": table, "k_pages": make((n_pages, hkv, b, d), **args), "v_pages": make((n_pages, hkv, b, d), **args)}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 12345)
    op, dt, hq, hkv, d = case["op"], _DT[case["dtype"]], case["hq"], case["hkv"], case["d"]
    s = {"op": op}
    if op != "attn":
        s["inv_freq"] = [float(case["base"]) ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
        s["pair_axis"], s["interleaved"] = _axes_of_pairs(case), bool(case["interleaved"])
    if op == "rope":
        n = case["tokens"]
        s.update(q=_rows(g, n, hq, d, dt), k=_rows(g, n, hkv, d, dt), positions=_positions(g, n, case["axes"]), inverse=bool(case["inverse"]))
    elif op == "append":
        starts, new = _append_lens(case)
        n = sum(new)
        s.update(_pages(g, case, [a + b for a, b in zip(starts, new)], False))
        s.update(q=_rows(g, n, hq, d, dt), k=_rows(g, n, hkv, d, dt), v=_rows(g, n, hkv, d, dt))
        s["start"], s["cu_new"] = torch.tensor(starts, dtype=torch.int32, device="cuda"), _cu(new)
        # text is where it is in its sequence; images have positions of their own
        s["positions"] = None if case["axes"] == 1 else _positions(g, n, case["axes"])
    else:
        nq, nk = _attn_lens(case)
        s.update(_pages(g, case, nk, True))
        s.update(q=_rows(g, sum(nq), hq, d, dt, 1.5), nq=nq, nk=nk, max_q=max(nq), max_len=max(nk), cu_q=_cu(nq))
        s["lens"] = torch.tensor(nk, dtype=torch.int32, device="cuda")
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _cos_sin(s, positions):
    """positions [axes, tokens] -> cosines and sines [tokens, 1, pairs], angles in 64 bits (far positions)."""
    freq = torch.tensor(s["inv_freq"], dtype=torch.float64, device=positions.device)
    axis = torch.tensor(s["pair_axis"], device=positions.device)
    angle = positions.double()[axis].T * freq
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _rotate(s, x, cos, sin):
    n = cos.shape[-1]
    f = x.float()
    a, b = (f[..., 0:2 * n:2], f[..., 1:2 * n:2]) if s["interleaved"] else (f[..., :n], f[..., n:2 * n])
    out = f.clone()
    if s["interleaved"]:
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = a * cos - b * sin, b * cos + a * sin
    else:
        out[..., :n], out[..., n:2 * n] = a * cos - b * sin, b * cos + a * sin
    return out.to(x.dtype)


def _plain_rope(s):
    cos, sin = _cos_sin(s, s["positions"])
    if s["inverse"]:
        sin = -sin
    return _rotate(s, s["q"], cos, sin), _rotate(s, s["k"], cos, sin)


def _plain_append(s):
    start, cu, b, total = s["start"].long(), s["cu_new"].long(), s["block"], s["k"].shape[0]
    seq = torch.repeat_interleave(torch.arange(start.shape[0], device=start.device), cu[1:] - cu[:-1], output_size=total)
    place = start[seq] + torch.arange(total, device=start.device) - cu[seq]
    cos, sin = _cos_sin(s, place[None] if s["positions"] is None else s["positions"])
    page = s["block_table"][seq, place // b].long()
    s["k_pages"][page, :, place % b] = _rotate(s, s["k"], cos, sin)
    s["v_pages"][page, :, place % b] = s["v"]
    return _rotate(s, s["q"], cos, sin), s["k_pages"], s["v_pages"]


def _plain_attn(s):
    q, b = s["q"], s["block"]
    hq, d, hkv = q.shape[1], q.shape[2], s["k_pages"].shape[1]
    out = torch.empty_like(q)
    lse = torch.empty((hq, q.shape[0]), dtype=torch.float32, device=q.device)
    q0 = 0
    for i, (nq, nk) in enumerate(zip(s["nq"], s["nk"])):
        page = s["block_table"][i, :-(-nk // b)].long()
        kk, vv = (s[w][page].transpose(0, 1).reshape(hkv, -1, d)[:, :nk].float() for w in ("k_pages", "v_pages"))
        step = max(1, (1 << 29) // (hq * nk))
        for r0 in range(0, nq, step):
            r = min(step, nq - r0)
            x = q[q0 + r0:q0 + r0 + r].float().view(r, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
            x = torch.matmul(x, kk.transpose(1, 2)).view(hq, r, nk).mul_(d ** -0.5)
            rows = torch.arange(r0, r0 + r, device=q.device)[:, None] + (nk - nq)
            x.masked_fill_(torch.arange(nk, device=q.device)[None] > rows, -math.inf)
            m = x.amax(-1, keepdim=True)
            p = torch.exp(x - m)
            l = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(hkv, -1, nk), vv).view(hq, r, d) / l
            out[q0 + r0:q0 + r0 + r] = o.transpose(0, 1).to(q.dtype)
            lse[:, q0 + r0:q0 + r0 + r] = (m + torch.log(l))[..., 0]
        q0 += nq
    return out, lse


def run(s):
    op = s["op"]
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn}[op](s)
    from paper_2608_05326_b200 import binding

    if op == "attn":
        cache = binding.Kv16Cache(s["k_pages"], s["v_pages"], s["block_table"])
        return cache.attn(s["q"], s["lens"], cu_q=s["cu_q"], max_q=s["max_q"], max_len=s["max_len"], return_lse=True)
    if "rotation" not in s:  # a model has one
        s["rotation"] = binding.Rotation(s["inv_freq"], axes=s["pair_axis"], interleaved=s["interleaved"])
    if op == "rope":
        return binding.qevict_rope(s["q"], s["positions"], s["rotation"], k=s["k"], inverse=s["inverse"])
    cache = binding.Kv16Cache(s["k_pages"], s["v_pages"], s["block_table"])
    q = cache.append(s["k"], s["v"], s["start"], cu_new=s["cu_new"], rotation=s["rotation"], positions=s["positions"], q=s["q"])
    return q, s["k_pages"], s["v_pages"]


# ---- work ---------------------------------------------------------------------------------------------------------
def work(case):
    op, hq, hkv, d = case["op"], case["hq"], case["hkv"], case["d"]
    if op == "attn":
        nq, nk = _attn_lens(case)
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(nq, nk))
        blocks = sum(-(-x // case["block"]) for x in nk)
        return {"bytes": 2 * d * (2 * sum(nq) * hq + 2 * sum(nk) * hkv) + 4 * sum(nq) * hq + 4 * blocks + 8 * case["n_seqs"], "flops": 4 * d * hq * pairs}
    n = case["tokens"] if op == "rope" else sum(_append_lens(case)[1])
    bytes_ = 4 * n * d * (hq + hkv * (2 if op == "append" else 1))
    if op == "rope" or case["axes"] > 1:
        bytes_ += 4 * n * case["axes"]
    if op == "append":
        bytes_ += 4 * sum((a + x - 1) // case["block"] - a // case["block"] + 1 for a, x in zip(*_append_lens(case))) + 8 * case["n_seqs"]
    return {"bytes": bytes_, "flops": 3 * n * case["rot"] * (hq + hkv)}


# ---- exact forms (64 bits) --------------------------------------------------------------------------------------
def _turn(case, x, pos, inverse=False):
    """x [tokens, heads, d], pos [axes, tokens]: each pair as a complex number times exp(i pos freq)."""
    n, x = case["rot"] // 2, x.double()
    freq = torch.exp(torch.arange(n, dtype=torch.float64, device=x.device) * (-2.0 / case["rot"] * math.log(case["base"])))
    theta = torch.stack([pos[a].double() for a in _axes_of_pairs(case)], dim=1) * freq * (-1.0 if inverse else 1.0)
    unit = torch.polar(torch.ones_like(theta), theta)[:, None]
    pair = x[..., :2 * n].unflatten(-1, (n, 2) if case["interleaved"] else (2, n))
    if not case["interleaved"]:
        pair = pair.transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * unit)
    if not case["interleaved"]:
        turned = turned.transpose(-1, -2)
    return torch.cat([turned.flatten(-2), x[..., 2 * n:]], dim=-1)


def _exact_append(case, s):
    starts, new = _append_lens(case)
    place = torch.cat([torch.arange(a, a + m, device="cuda") for a, m in zip(starts, new)])
    pos = place[None] if s["positions"] is None else s["positions"]
    k, b, row = _turn(case, s["k"], pos), case["block"], 0
    pools = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
    for i, (a, m) in enumerate(zip(starts, new)):
        pages = s["block_table"][i, a // b:(a + m - 1) // b + 1].long()
        for w, rows in (("k", k[row:row + m]), ("v", s["v"][row:row + m].double())):
            span = pools[w][pages].transpose(1, 2).flatten(0, 1)  # [tokens, hkv, d]
            span[a % b:a % b + m] = rows
            pools[w][pages] = span.unflatten(0, (-1, b)).transpose(1, 2)
        row += m
    return _turn(case, s["q"], pos), pools["k"], pools["v"]


def _exact_attn(case, s):
    q, b, group = s["q"], case["block"], case["hq"] // case["hkv"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.zeros((case["hq"], q.shape[0]), dtype=torch.float64, device=q.device)
    q0 = 0
    for s_i, (nq, nk) in enumerate(zip(*_attn_lens(case))):
        pages = s["block_table"][s_i, :-(-nk // b)].long()
        for h in range(case["hkv"]):
            k, v = (s[w][pages, h].flatten(0, 1)[:nk].double() for w in ("k_pages", "v_pages"))
            for r0 in range(0, nq, 1024):
                e = min(nq, r0 + 1024)
                hidden = torch.arange(nk, device=q.device)[None] > torch.arange(r0, e, device=q.device)[:, None] + nk - nq
                for g in range(h * group, (h + 1) * group):
                    z = ((q[q0 + r0:q0 + e, g].double() @ k.T) / math.sqrt(case["d"])).masked_fill_(hidden, -math.inf)
                    l = torch.logsumexp(z, dim=-1)
                    out[q0 + r0:q0 + e, g] = torch.exp(z - l[:, None]) @ v
                    lse[g, q0 + r0:q0 + e] = l
        q0 += nq
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return tuple(_turn(case, s[w], s["positions"], s["inverse"]) for w in ("q", "k"))
    return {"append": _exact_append, "attn": _exact_attn}[case["op"]](case, s)
