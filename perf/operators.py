"""Prompt attention and the 8-bit block-scaled cache (append, attention, eviction): cases, plain forms, exact forms.

Shapes are those of the decode workloads of this library (Llama-3-8B: 32 / 8 heads of 128; Qwen2.5-7B: 28 / 4 heads of
128; the tiny test shapes with heads of 64) and their contexts (2k to 128k), window sizes 32 and 64 as block sizes.

Every case is one call; `op` says which:

  prompt  causal attention over packed prompts.  `n_seqs` sequences, the longest of `max_q` new tokens behind a prefix of
          `prefix` tokens that are already there (a prompt given in pieces); prefix 0: whole prompts.
  attn    one token per sequence over the 8-bit cache, with the accumulated attention mass of every block.
  append  new tokens into the 8-bit cache: one per sequence (`max_new` 1) or prompt pieces that start on a block boundary.
  evict   table, scores and lengths after dropping all but the `budget` best blocks.
"""

import math
import random

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_HEADS = [(32, 8, 128), (28, 4, 128), (8, 8, 64), (4, 2, 64), (16, 1, 128)]


# ---- cases ----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one short question on a small model: latency of a single launch
        dict(name="prompt-short", op="prompt", hq=4, hkv=2, d=64, dtype="fp16", n_seqs=1, max_q=77, prefix=0, ragged=0),
        # a batch of prompts of very different lengths, packed without padding
        dict(name="prompt-packed", op="prompt", hq=32, hkv=8, d=128, dtype="bf16", n_seqs=12, max_q=4001, prefix=0, ragged=1),
        # the 32k prompt of the headline workload, in one piece
        dict(name="prompt-32k", op="prompt", hq=32, hkv=8, d=128, dtype="bf16", n_seqs=1, max_q=32768, prefix=0, ragged=0),
        # a piece of 500 tokens of a long prompt whose first 16k tokens are already there
        dict(name="prompt-piece", op="prompt", hq=28, hkv=4, d=128, dtype="fp16", n_seqs=2, max_q=500, prefix=16000, ragged=1),
        # one user, short context: the smallest decode step
        dict(name="attn-small", op="attn", hq=32, hkv=8, d=128, dtype="bf16", code="int8", block=64, n_seqs=1, max_len=2048, ragged=0),
        # a server's batch of ragged contexts
        dict(name="attn-batch", op="attn", hq=32, hkv=8, d=128, dtype="bf16", code="int8", block=64, n_seqs=16, max_len=32768, ragged=1),
        # 8 long documents, floating 8-bit codes
        dict(name="attn-64k", op="attn", hq=28, hkv=4, d=128, dtype="fp16", code="e4m3", block=32, n_seqs=8, max_len=65536, ragged=0),
        # one token for each of 16 sequences (one in 64 fills its block)
        dict(name="append-token", op="append", hkv=8, d=128, dtype="bf16", code="int8", block=64, n_seqs=16, max_start=32768, max_new=1),
        # four prompts at once into an empty cache
        dict(name="append-prompts", op="append", hkv=8, d=128, dtype="bf16", code="int8", block=64, n_seqs=4, max_start=0, max_new=16001),
        # the next piece of 12 prompts, floating codes
        dict(name="append-pieces", op="append", hkv=4, d=128, dtype="fp16", code="e4m3", block=32, n_seqs=12, max_start=8192, max_new=2048),
        # one sequence over its budget
        dict(name="evict-one", op="evict", block=32, n_seqs=1, max_blocks=1024, budget=192, sink=1, recent=4, ragged=0),
        # a batch of long sequences
        dict(name="evict-batch", op="evict", block=16, n_seqs=16, max_blocks=8192, budget=2000, sink=1, recent=8, ragged=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "attn", "attn", "append", "evict"])
    hq, hkv, d = rng.choice(_HEADS)
    dtype, code, block = rng.choice(["bf16", "fp16"]), rng.choice(["int8", "e4m3"]), rng.choice([16, 32, 64, 128])
    if op == "prompt":
        max_q = _log(rng, 1, 16384)
        prefix = _log(rng, 1, 16384) if rng.random() < 0.4 else 0
        n = max(1, min(_log(rng, 1, 16), int(2.0e8 / (max_q * (prefix + max_q)))))
        return dict(op=op, hq=hq, hkv=hkv, d=d, dtype=dtype, n_seqs=n, max_q=max_q, prefix=prefix, ragged=int(rng.random() < 0.7), pick=rng.randrange(1 << 30))
    if op == "attn":
        max_len = _log(rng, 1, 131072)
        n = max(1, min(_log(rng, 1, 64), 524288 // max_len))
        return dict(op=op, hq=hq, hkv=hkv, d=d, dtype=dtype, code=code, block=block, n_seqs=n, max_len=max_len, ragged=int(rng.random() < 0.7), pick=rng.randrange(1 << 30))
    if op == "append":
        max_new = 1 if rng.random() < 0.4 else _log(rng, 2, 16384)
        n = max(1, min(_log(rng, 1, 64), 65536 // max_new))
        return dict(op=op, hkv=hkv, d=d, dtype=dtype, code=code, block=block, n_seqs=n, max_start=rng.choice([0, _log(rng, 1, 16384)]), max_new=max_new, pick=rng.randrange(1 << 30))
    mb = _log(rng, 8, 8192)
    sink, recent = rng.randrange(0, 3), rng.randrange(0, 3)
    return dict(op=op, block=block, n_seqs=_log(rng, 1, 64), max_blocks=mb, budget=rng.randrange(sink + recent, mb + 1), sink=sink, recent=recent, ragged=int(rng.random() < 0.7), pick=rng.randrange(1 << 30))


def _lens(case, longest, least=1):
    """Lengths of the sequences: the first is the longest; the others are spread below it where the case is ragged."""
    rng = random.Random(case.get("pick", 7))
    rest = case["n_seqs"] - 1
    return [longest] + [rng.randint(min(least, longest), longest) if case.get("ragged", 1) else longest for _ in range(rest)]


def _prompt_lens(case):
    nq = _lens(case, case["max_q"])
    return nq, [n + p for n, p in zip(nq, _lens(dict(case, pick=case.get("pick", 7) + 1), case["prefix"], 0))]


def _append_lens(case):
    starts = _lens(case, case["max_start"], 0)
    if case["max_new"] == 1:
        return starts, [1] * case["n_seqs"]
    # prompt pieces start on a block boundary
    return [s // case["block"] * case["block"] for s in starts], _lens(dict(case, pick=case.get("pick", 7) + 1), case["max_new"])


def _cu(lens, dev):
    return torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=dev)


# ---- the quantizer of the cache (definition) ----------------------------------------------------------------------
def _quantize(x, code):
    """x [..., B, d] float32 -> codes of the block, scale [...]: scale = amax / 127 (or / 448), code = nearest of x / scale."""
    amax = x.abs().amax(dim=(-2, -1))
    scale = amax / torch.full_like(amax, 127.0 if code == "int8" else 448.0)  # a true division: by a plain number it is a product
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    y = x / scale[..., None, None]
    if code == "int8":
        return torch.round(y).clamp(-127, 127).to(torch.int8), scale
    return y.clamp(-448, 448).to(torch.float8_e4m3fn), scale


# ---- inputs -----------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 12345)
    return g


def _cache(case, lens, g, filled):
    """Pools with room for every sequence, pages handed out in a shuffled order; filled: prompts quantized into them."""
    dt, b, n, hkv, d = _DT[case["dtype"]], case["block"], case["n_seqs"], case["hkv"], case["d"]
    mb = max(1, -(-(max(lens) + 1) // b))
    cdt = torch.int8 if case["code"] == "int8" else torch.float8_e4m3fn
    per = [max(1, -(-(x + 1) // b)) for x in lens]
    n_pages = sum(per) + 3
    perm = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((n, mb), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(mb, device="cuda")[None] + torch.tensor([sum(per[:i]) for i in range(n)], device="cuda")[:, None]
    used = torch.arange(mb, device="cuda")[None] < torch.tensor(per, device="cuda")[:, None]
    table[used] = perm[at[used]]
    s = {"block": b, "code": case["code"], "max_len": max(lens), "block_table": table,
         "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    gain = torch.exp(0.5 * torch.randn((1, hkv, 1, d), generator=g, device="cuda"))  # channels differ in size
    for w in "kv":
        codes = torch.zeros((n_pages, hkv, b, d), dtype=cdt, device="cuda")
        scale = torch.zeros((n_pages, hkv), dtype=torch.float32, device="cuda")
        if filled:
            step = max(1, (1 << 27) // (hkv * b * d))
            for p in range(0, n_pages, step):
                x = (torch.randn((min(step, n_pages - p), hkv, b, d), generator=g, device="cuda") * gain).to(dt).float()
                codes[p:p + step], scale[p:p + step] = _quantize(x, case["code"])
        s[w + "_codes"], s[w + "_scale"] = codes, scale
        s[w + "_tail"] = torch.randn((n, hkv, b, d), generator=g, device="cuda").to(dt)
    return s


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"op": op}
    if op == "prompt":
        nq, nk = _prompt_lens(case)
        dt = _DT[case["dtype"]]
        s["q"] = torch.randn((sum(nq), case["hq"], case["d"]), generator=g, device="cuda").mul_(1.5).to(dt)
        s["k"] = torch.randn((sum(nk), case["hkv"], case["d"]), generator=g, device="cuda").to(dt)
        s["v"] = torch.randn((sum(nk), case["hkv"], case["d"]), generator=g, device="cuda").to(dt)
        s["cu_q"], s["cu_k"] = _cu(nq, "cuda"), _cu(nk, "cuda")
        s["nq"], s["nk"] = nq, nk
        s["max_q"], s["max_k"] = max(nq), max(nk)
    elif op == "attn":
        lens = _lens(case, case["max_len"])
        s.update(_cache(case, lens, g, True))
        s["q"] = torch.randn((case["n_seqs"], case["hq"], case["d"]), generator=g, device="cuda").mul_(1.5).to(_DT[case["dtype"]])
        s["scores"] = torch.rand(s["block_table"].shape, generator=g, device="cuda")
    elif op == "append":
        starts, new = _append_lens(case)
        s.update(_cache(case, [a + b for a, b in zip(starts, new)], g, False))
        dt = _DT[case["dtype"]]
        gain = torch.exp(0.5 * torch.randn((1, case["hkv"], case["d"]), generator=g, device="cuda"))
        s["k"] = (torch.randn((sum(new), case["hkv"], case["d"]), generator=g, device="cuda") * gain).to(dt)
        s["v"] = (torch.randn((sum(new), case["hkv"], case["d"]), generator=g, device="cuda") * gain).to(dt)
        s["start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["cu_new"], s["max_new"] = _cu(new, "cuda"), max(new)
    else:
        n, mb, b = case["n_seqs"], case["max_blocks"], case["block"]
        full = _lens(case, mb - 1)
        s["lens"] = torch.tensor([f * b + (5 * i) % b for i, f in enumerate(full)], dtype=torch.int32, device="cuda")
        s["block_table"] = torch.randperm(n * mb, generator=g, device="cuda").to(torch.int32).view(n, mb)
        # masses are heavy-tailed; many late blocks have the same small one
        x = torch.exp(2.0 * torch.randn((n, mb), generator=g, device="cuda"))
        s["scores"] = torch.where(torch.rand((n, mb), generator=g, device="cuda") < 0.3, torch.full_like(x, 0.25), x)
        s.update(block=b, n_pages=n * mb, budget=case["budget"], sink=case["sink"], recent=case["recent"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _softmax_parts(x):
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(x - m)
    return p, p.sum(-1, keepdim=True), m


def _plain_prompt(s):
    q, k, v = s["q"], s["k"], s["v"]
    hq, d, hkv = q.shape[1], q.shape[2], k.shape[1]
    out = torch.empty_like(q)
    lse = torch.empty((hq, q.shape[0]), dtype=torch.float32, device=q.device)
    q0 = k0 = 0
    for nq, nk in zip(s["nq"], s["nk"]):
        kk = k[k0:k0 + nk].float().permute(1, 2, 0)
        vv = v[k0:k0 + nk].float().transpose(0, 1)
        step = max(1, (1 << 29) // (hq * nk))
        for i in range(0, nq, step):
            r = min(step, nq - i)
            x = q[q0 + i:q0 + i + r].float().view(r, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
            x = torch.matmul(x, kk).view(hq, r, nk).mul_(d ** -0.5)
            rows = torch.arange(i, i + r, device=q.device)[:, None] + (nk - nq)
            x.masked_fill_(torch.arange(nk, device=q.device)[None] > rows, -math.inf)
            p, l, m = _softmax_parts(x)
            o = torch.matmul(p.view(hkv, -1, nk), vv).view(hq, r, d) / l
            out[q0 + i:q0 + i + r] = o.transpose(0, 1).to(q.dtype)
            lse[:, q0 + i:q0 + i + r] = (m + torch.log(l))[..., 0]
        q0, k0 = q0 + nq, k0 + nk
    return out, lse


def _plain_rows(s, w, lens):
    """Keys or values of the cache as float32 [n, hkv, max_blocks * block, d]."""
    table, b = s["block_table"], s["block"]
    n, mb = table.shape
    page = table.clamp(min=0).long()
    x = s[w + "_codes"][page].float() * s[w + "_scale"][page][..., None, None]  # [n, mb, hkv, b, d]
    open_block = (lens // b).clamp(max=mb - 1).long()
    is_open = ((torch.arange(mb, device=x.device)[None] == open_block[:, None]) & (lens % b > 0)[:, None])[..., None, None, None]
    x = torch.where(is_open, s[w + "_tail"].float()[:, None], x)
    return x.transpose(1, 2).reshape(n, x.shape[2], mb * b, x.shape[-1])


def _plain_attn(s):
    q, lens, b = s["q"], s["lens"], s["block"]
    n, hq, d = q.shape
    mb = s["block_table"].shape[1]
    hkv = s["k_codes"].shape[1]
    x = torch.matmul(q.float().view(n, hkv, hq // hkv, d), _plain_rows(s, "k", lens).transpose(-1, -2)) * d ** -0.5
    x.masked_fill_((torch.arange(mb * b, device=q.device)[None] >= lens[:, None])[:, None, None], -math.inf)
    p, l, m = _softmax_parts(x)
    out = torch.matmul(p, _plain_rows(s, "v", lens)) / l
    mass = (p / l).sum((1, 2)).view(n, mb, b).sum(-1)
    return out.view(n, hq, d).to(q.dtype), (m + torch.log(l)).view(n, hq), s["scores"] + mass


def _plain_append(s):
    b, start, cu = s["block"], s["start"].long(), s["cu_new"].long()
    n = start.shape[0]
    new = cu[1:] - cu[:-1]
    total = s["k"].shape[0]
    seq = torch.repeat_interleave(torch.arange(n, device=start.device), new, output_size=total)
    pos = start[seq] + torch.arange(total, device=start.device) - cu[seq]
    first = start // b
    done = (start + new) // b - first  # blocks of each sequence that are complete now
    most = -(-s["max_new"] // b) + 1
    j = torch.arange(most, device=start.device)
    page = s["block_table"].gather(1, (first[:, None] + j[None]).clamp(max=s["block_table"].shape[1] - 1)).long()
    full = j[None] < done[:, None]
    at = pos - first[seq] * b
    for w in "kv":
        tail = s[w + "_tail"]
        x = torch.zeros((n, most * b) + tail.shape[1:2] + tail.shape[3:], dtype=tail.dtype, device=tail.device)
        x[:, :b] = tail.transpose(1, 2)
        x[seq, at] = s[w]
        x = x.view(n, most, b, tail.shape[1], tail.shape[3]).transpose(2, 3)
        codes, scale = _quantize(x[full].float(), s["code"])
        s[w + "_codes"][page[full]] = codes
        s[w + "_scale"][page[full]] = scale
        rows = (pos // b) == ((start + new) // b)[seq]  # tokens of the block that stays open
        tail[seq[rows], :, pos[rows] % b] = s[w][rows]
    return tuple(s[w + x] for w in "kv" for x in ("_codes", "_scale", "_tail"))


def _plain_evict(s):
    table, scores, lens, b = s["block_table"], s["scores"], s["lens"].long(), s["block"]
    n, mb = table.shape
    full = lens // b
    i = torch.arange(mb, device=table.device)[None].expand(n, mb)
    over = (full > s["budget"])[:, None]
    middle = (i >= s["sink"]) & (i < (full - s["recent"])[:, None])
    order = torch.sort(torch.nan_to_num(scores, nan=-math.inf), dim=1, descending=True, stable=True)[1]
    order = order.gather(1, torch.sort(middle.gather(1, order).int(), dim=1, descending=True, stable=True)[1])
    rank = torch.empty_like(order).scatter_(1, order, i)
    gone = over & middle & (rank >= s["budget"] - s["sink"] - s["recent"])
    keep = ~gone
    to = torch.where(keep, keep.long().cumsum(1) - 1, mb)
    pad = lambda fill, x: torch.full((n, mb + 1), fill, dtype=x.dtype, device=x.device).scatter_(1, to, x)[:, :mb]  # noqa: E731
    freed_to = torch.where(gone, gone.long().cumsum(1) - 1, mb)
    freed = torch.full((n, mb + 1), -1, dtype=torch.int32, device=table.device).scatter_(1, freed_to, table)[:, :mb]
    n_gone = gone.sum(1)
    # entries behind the kept ones: the scatter leaves the fill value, the last one is dropped with column mb
    return {"block_table": pad(-1, table), "lens": (lens - n_gone * b).int(), "scores": pad(0.0, scores),
            "kept": pad(-1, i.int()), "freed": freed, "n_freed": n_gone.int()}


def run(s):
    op = s["op"]
    if not own:
        return {"prompt": _plain_prompt, "attn": _plain_attn, "append": _plain_append, "evict": _plain_evict}[op](s)
    from paper_2608_05326_b200 import binding

    if op == "prompt":
        return binding.qevict_prompt_attn(s["q"], s["k"], s["v"], cu_q=s["cu_q"], cu_k=s["cu_k"], max_q=s["max_q"], max_k=s["max_k"], return_lse=True)
    if op == "evict":
        return binding.qevict_kv8_evict(s["block_table"], s["lens"], s["scores"], block=s["block"], n_pages=s["n_pages"], budget=s["budget"], sink=s["sink"], recent=s["recent"])
    cache = binding.Kv8Cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"], s["block_table"])
    if op == "attn":
        return cache.attn(s["q"], s["lens"], max_len=s["max_len"], scores=s["scores"], return_lse=True)
    cache.append(s["k"], s["v"], s["start"], cu_new=s["cu_new"], max_new=s["max_new"])
    return tuple(s[w + x] for w in "kv" for x in ("_codes", "_scale", "_tail"))


# ---- work ---------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "prompt":
        nq, nk = _prompt_lens(case)
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(nq, nk))
        return {"bytes": 2 * case["d"] * (2 * sum(nq) * case["hq"] + 2 * sum(nk) * case["hkv"]) + 4 * sum(nq) * case["hq"],
                "flops": 4 * case["d"] * case["hq"] * pairs}
    if op == "attn":
        lens = _lens(case, case["max_len"])
        rows = case["hkv"] * case["d"]
        whole = sum(x // case["block"] * case["block"] for x in lens)
        blocks = sum(-(-x // case["block"]) for x in lens)
        return {"bytes": 2 * whole * rows + 4 * (sum(lens) - whole) * rows + blocks * (8 * case["hkv"] + 12) + case["n_seqs"] * case["hq"] * (4 * case["d"] + 4),
                "flops": 4 * sum(lens) * case["hq"] * case["d"]}
    if op == "append":
        starts, new = _append_lens(case)
        b, row = case["block"], case["hkv"] * case["d"]
        done = sum((a + x) // b - a // b for a, x in zip(starts, new))
        left = sum(min(x, (a + x) % b) for a, x in zip(starts, new))
        old = sum(a % b for a, x in zip(starts, new) if (a + x) // b > a // b)
        return {"bytes": 2 * row * (2 * sum(new) + 2 * old + done * b + 2 * left) + 8 * done * case["hkv"] + 4 * done, "flops": 2 * 2 * row * b * done}
    n, mb = case["n_seqs"], case["max_blocks"]
    return {"bytes": n * (mb * (4 + 4) + 4 + 4 * (4 * mb + 2)), "flops": n * mb}


# ---- exact forms (64 bits) --------------------------------------------------------------------------------------
def _exact_heads(q, k, v, allowed):
    """q [r, d], k, v [n, d], allowed [r, n] -> out [r, d], lse [r], probabilities [r, n], all float64."""
    z = (q @ k.T) / math.sqrt(q.shape[-1])
    z = torch.where(allowed, z, torch.full_like(z, -math.inf))
    lse = torch.logsumexp(z, dim=-1)
    p = torch.exp(z - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    return p @ v, lse, p


def _exact_prompt(case, s):
    q, k, v = s["q"], s["k"], s["v"]
    group = case["hq"] // case["hkv"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.zeros((case["hq"], q.shape[0]), dtype=torch.float64, device=q.device)
    q0 = k0 = 0
    for nq, nk in zip(*_prompt_lens(case)):
        for h in range(case["hq"]):
            kh, vh = k[k0:k0 + nk, h // group].double(), v[k0:k0 + nk, h // group].double()
            for i in range(0, nq, 4096):
                e = min(nq, i + 4096)
                ok = torch.arange(nk, device=q.device)[None] <= torch.arange(i, e, device=q.device)[:, None] + nk - nq
                out[q0 + i:q0 + e, h], lse[h, q0 + i:q0 + e], _ = _exact_heads(q[q0 + i:q0 + e, h].double(), kh, vh, ok)
        q0, k0 = q0 + nq, k0 + nk
    return out, lse


def _exact_attn(case, s):
    n, hq, d = s["q"].shape
    hkv, b, mb = case["hkv"], case["block"], s["block_table"].shape[1]
    out = torch.zeros((n, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((n, hq), dtype=torch.float64, device="cuda")
    scores = s["scores"].double().clone()
    for i, ln in enumerate(_lens(case, case["max_len"])):
        pages = s["block_table"][i, :ln // b].long()
        for h in range(hkv):
            rows = {}
            for w in "kv":
                x = (s[w + "_codes"][pages, h].double() * s[w + "_scale"][pages, h].double()[:, None, None]).reshape(-1, d)
                rows[w] = torch.cat([x, s[w + "_tail"][i, h, :ln % b].double()])
            hs = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            ok = torch.ones((hq // hkv, ln), dtype=torch.bool, device="cuda")
            out[i, hs], lse[i, hs], p = _exact_heads(s["q"][i, hs].double(), rows["k"], rows["v"], ok)
            per = torch.zeros(mb * b, dtype=torch.float64, device="cuda")
            per[:ln] = p.sum(0)
            scores[i] += per.view(mb, b).sum(1)
    return out, lse, scores


def _exact_append(case, s):
    """The definition rounds the scale and the quotient to 32 bits; a quotient of 64 bits rounded once more is the same."""
    got = []
    most, b = (127.0 if case["code"] == "int8" else 448.0), case["block"]
    starts, new = _append_lens(case)
    for w in "kv":
        codes, scale, tail = s[w + "_codes"].double(), s[w + "_scale"].double(), s[w + "_tail"].double()
        row = 0
        for i, (a, m) in enumerate(zip(starts, new)):
            x = torch.cat([tail[i, :, :a % b], s[w][row:row + m].double().transpose(0, 1)], dim=1)  # [hkv, tokens, d]
            row += m
            whole = x.shape[1] // b
            if whole:
                pages = s["block_table"][i, a // b:a // b + whole].long()
                y = x[:, :whole * b].reshape(case["hkv"], whole, b, -1).transpose(0, 1)
                sc = (y.abs().amax((2, 3)) / most).float().double()
                sc = torch.where(sc > 0, sc, torch.ones_like(sc))
                y = (y / sc[..., None, None]).float()
                codes[pages] = (torch.round(y) if case["code"] == "int8" else y.to(torch.float8_e4m3fn)).double()
                scale[pages] = sc
            left = x.shape[1] - whole * b
            tail[i, :, :left] = x[:, whole * b:]
        got += [codes if case["code"] == "e4m3" else codes.to(torch.int8), scale, tail]
    return tuple(got)


def exact(case, seed):
    if case["op"] == "evict":
        return None  # whole numbers, and scores that are only moved
    s = prepare(case, seed)
    return {"prompt": _exact_prompt, "attn": _exact_attn, "append": _exact_append}[case["op"]](case, s)
