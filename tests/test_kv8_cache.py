"""The 8-bit block-scaled cache: append, attention with block masses, eviction, and a run of them together."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8 as oracle
from oracle import prompt as po
from paper_2608_05326_b200 import binding

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


# ---- the oracle's quantizer -----------------------------------------------------------------------------------
def test_oracle_e4m3_rounding_is_the_formats():
    y = np.concatenate([np.linspace(-460, 460, 20001), np.linspace(-0.05, 0.05, 5001), oracle.e4m3_values()])
    mids = (oracle.e4m3_values()[1:] + oracle.e4m3_values()[:-1]) / 2
    y = np.concatenate([y, mids, -mids]).astype(np.float32)
    want = torch.from_numpy(y).clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.round_e4m3(y.astype(np.float64)), want)


def test_oracle_quantizer_by_hand():
    x = np.zeros((2, 2))
    assert oracle.quantize(x, "int8") [1] == 1.0
    x = np.array([[254.0, 3.0], [1.0, -254.0]])  # scale 2: 1.5 and 0.5 are ties
    v, s = oracle.quantize(x, "int8")
    assert s == 2.0 and v.tolist() == [[127.0, 2.0], [0.0, -127.0]]
    v, s = oracle.quantize(np.array([[1.0, np.nan]]), "int8")
    assert s == 1.0 and (v == 0).all()


def test_oracle_eviction_by_hand():
    t = np.array([[10, 11, 12, 13, 14, 15, -1]], np.int32)
    sc = np.array([[0.0, 2.0, 5.0, 2.0, np.nan, 1.0, 0.5]], np.float32)
    got = oracle.evict(t, np.array([6 * 16 + 3]), sc, 16, 100, 4, 1, 1)
    assert got["block_table"].tolist() == [[10, 11, 12, 15, -1, -1, -1]] and got["kept"].tolist() == [[0, 1, 2, 5, 6, -1, -1]]
    assert got["freed"][0, :2].tolist() == [13, 14] and got["lens"][0] == 4 * 16 + 3 and got["n_freed"][0] == 2


# ---- refusals: checked before anything reaches a device -------------------------------------------------------
def _view(**over):
    c = binding.qevict_kv8_cache()
    values = dict(struct_size=C.sizeof(c), device=0, dtype=1, code=0, n_seqs=2, n_kv_heads=2, head_dim=64, block=32, max_blocks=8, n_pages=16,
                  k_codes=4096, v_codes=4096, k_scale=4096, v_scale=4096, k_tail=4096, v_tail=4096, block_table=4096)
    values.update(over)
    for n, x in values.items():
        setattr(c, n, x)
    return c


def _append(view, k=4096, v=4096, ts=128, hs=64, total=4, start=4096, cu=4096, max_new=4):
    return binding.lib().qevict_kv8_append(C.byref(view), k, v, ts, hs, total, start, cu, max_new, None)


def _attn(view, hq=4, scale=0.0, q=4096, lens=4096, max_len=256, out=4096, lse=None, si=None, so=None, scratch=4096, n=1 << 40):
    return binding.lib().qevict_kv8_attn(C.byref(view), hq, scale, q, lens, max_len, out, lse, si, so, scratch, n, None)


def _evict(**over):
    a = binding.qevict_kv8_evict_args()
    values = dict(struct_size=C.sizeof(a), device=0, n_seqs=2, max_blocks=8, block=32, n_pages=16, budget=4, sink=1, recent=1, table=4096,
                  lens=4096, scores=4096, table_out=4096, lens_out=4096, scores_out=4096)
    values.update(over)
    for n, x in values.items():
        setattr(a, n, x)
    return binding.lib().qevict_kv8_evict(C.byref(a), None)


@pytest.mark.parametrize("over,status,word", [
    (dict(struct_size=4), 1, "struct_size"), (dict(device=-2), 1, "device"), (dict(dtype=5), 1, "dtype"), (dict(code=2), 1, "code"),
    (dict(n_seqs=-1), 1, "n_seqs"), (dict(head_dim=80), 4, "head_dim"), (dict(block=48), 4, "block"), (dict(n_kv_heads=0), 1, "n_kv_heads"),
    (dict(k_codes=None), 1, "NULL"), (dict(v_scale=None), 1, "NULL"), (dict(k_tail=None), 1, "NULL"), (dict(block_table=None), 1, "NULL"),
    (dict(k_codes=4104), 1, "aligned"), (dict(v_tail=4100), 1, "aligned"), (dict(k_scale=4097), 1, "aligned"), (dict(max_blocks=1 << 30), 4, "2^30"), (dict(n_pages=2 ** 30 + 1), 4, "n_pages"),
])
def test_unusable_caches_are_refused_with_a_reason(over, status, word):
    for st in (_append(_view(**over)), _attn(_view(**over))):
        assert st == status and word in binding.lib().qevict_last_error(None).decode()


@pytest.mark.parametrize("call,status,word", [
    (lambda: _append(_view(), total=-1), 1, "total_new"), (lambda: _append(_view(), cu=None, max_new=2), 1, "one token"),
    (lambda: _append(_view(), cu=None, max_new=1, total=1), 1, "n_seqs"), (lambda: _append(_view(), k=None), 1, "NULL"),
    (lambda: _append(_view(), start=None), 1, "NULL"), (lambda: _append(_view(), ts=100), 1, "16 bytes"), (lambda: _append(_view(), hs=-64), 1, "strides"),
    (lambda: _append(_view(), cu=4097), 1, "aligned"),
    (lambda: _attn(_view(), hq=3), 1, "multiple"), (lambda: _attn(_view(), hq=34), 4, "16 query heads"), (lambda: _attn(_view(), max_len=-1), 1, "max_len"),
    (lambda: _attn(_view(), scale=float("inf")), 1, "softmax_scale"), (lambda: _attn(_view(), scale=1e-40), 1, "softmax_scale"), (lambda: _attn(_view(), q=None), 1, "NULL"), (lambda: _attn(_view(), scratch=None), 1, "NULL"),
    (lambda: _attn(_view(), n=16), 3, "scratch"), (lambda: _attn(_view(), si=4096), 1, "score_out"), (lambda: _attn(_view(), q=4100), 1, "aligned"),
    (lambda: _attn(_view(n_seqs=8192, max_blocks=1 << 24), max_len=1 << 29), 4, "too large"),
    (lambda: _evict(struct_size=3), 1, "struct_size"), (lambda: _evict(budget=1), 1, "budget"), (lambda: _evict(max_blocks=20000), 4, "16384"),
    (lambda: _evict(table=None), 1, "NULL"), (lambda: _evict(freed=4096), 1, "together"), (lambda: _evict(lens=4097), 1, "aligned"), (lambda: _evict(block=0), 1, "block"),
])
def test_unusable_arguments_are_refused_with_a_reason(call, status, word):
    assert call() == status and word in binding.lib().qevict_last_error(None).decode()


@pytest.mark.parametrize("scale", [3e38, 2.5e38, float("nan"), -1e-3, 1e-31])
def test_scales_that_are_no_float_times_log2_e_are_refused(scale):
    assert _attn(_view(), scale=scale) == 1 and "softmax_scale" in binding.lib().qevict_last_error(None).decode()


def test_nothing_to_do_is_fine_without_a_device():
    empty = _view(n_seqs=0, k_tail=None, v_tail=None, block_table=None)
    assert _append(empty) == 0 and _attn(empty) == 0 and _evict(n_seqs=0) == 0
    assert _append(_view(), max_new=0) == 0 and _append(_view(), total=0) == 0


def test_scratch_grows_with_the_scores_asked_for():
    lib, a, b = binding.lib(), C.c_uint64(), C.c_uint64()
    binding._check(lib.qevict_kv8_attn_scratch_bytes(C.byref(_view()), 4, 256, 0, C.byref(a)))
    binding._check(lib.qevict_kv8_attn_scratch_bytes(C.byref(_view()), 4, 256, 1, C.byref(b)))
    assert 0 < a.value < b.value


# ---- a cache on both sides --------------------------------------------------------------------------------------
class Pair:
    """The same cache for the library and for the oracle; pages handed out in a shuffled order, pools poisoned."""

    def __init__(self, n_seqs, max_blocks, hkv, d, block, dtype, code, seed=0):
        self.n, self.hkv, self.d, self.block, self.dtype, self.code = n_seqs, hkv, d, block, dtype, code
        self.g = torch.Generator().manual_seed(seed)
        self.n_pages = n_seqs * max_blocks + 2
        table = torch.randperm(self.n_pages, generator=self.g)[:n_seqs * max_blocks].int().view(n_seqs, max_blocks)
        c = binding.Kv8Cache.allocate(self.n_pages, n_seqs, max_blocks, hkv, d, block, dtype, CODES[code])
        c.block_table.copy_(table)
        c.k_scale.fill_(float("nan"))
        c.v_scale.fill_(float("nan"))
        c.k_tail.fill_(float("nan"))
        c.v_tail.fill_(float("nan"))
        self.cache = c
        pool = (self.n_pages, hkv, block, d)
        self.o = oracle.Cache([np.zeros(pool) for _ in range(2)], [np.full(pool[:2], np.nan, np.float32) for _ in range(2)],
                              [np.full((n_seqs, hkv, block, d), np.nan) for _ in range(2)], table.numpy(), code)
        self.lens = np.zeros(n_seqs, np.int64)

    def random(self, total, gain=1.0):
        ch = torch.exp(0.5 * torch.randn((1, self.hkv, self.d), generator=self.g))
        return [(gain * ch * torch.randn((total, self.hkv, self.d), generator=self.g)).to(self.dtype) for _ in range(2)]

    def append(self, counts, kv=None, single=False, start=None, stream=None):
        start = self.lens if start is None else np.array(start)
        k, v = self.random(int(sum(counts))) if kv is None else kv
        cu = np.concatenate([[0], np.cumsum(counts)])
        self.o.append([x.double().numpy() for x in (k, v)], start, counts, cu[:-1])
        dev = dict(dtype=torch.int32, device="cuda")
        if single:
            self.cache.append(k.cuda(), v.cuda(), torch.tensor(start, **dev), stream=stream)
        else:
            self.cache.append(k.cuda(), v.cuda(), torch.tensor(start, **dev), torch.tensor(cu, **dev), max(1, max(counts)), stream=stream)
        self.lens = np.where(np.array(start) >= 0, start + np.array(counts), self.lens)

    def check_state(self):
        for w, (codes, scale, tail) in enumerate(((self.cache.k_codes, self.cache.k_scale, self.cache.k_tail), (self.cache.v_codes, self.cache.v_scale, self.cache.v_tail))):
            same = [np.array_equal(codes.float().cpu().numpy().astype(np.float64), self.o.codes[w]),
                    np.array_equal(scale.cpu().numpy(), self.o.scale[w], equal_nan=True)]
            tail = tail.double().cpu().numpy()
            for s in range(self.n):  # rows of the open block; the others hold whatever was there
                m = min(int(self.lens[s]), self.o.table.shape[1] * self.block) % self.block
                same.append(np.array_equal(tail[s, :, :m], self.o.tail[w][s, :, :m], equal_nan=True))
            assert all(same), (w, same)

    def attend(self, hq, lens=None, scores=None, max_len=None, scale=0.0, gain=1.0, expect=None):
        lens = self.lens if lens is None else np.array(lens)
        q = (gain * torch.randn((self.n, hq, self.d), generator=self.g)).to(self.dtype)
        dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
        out, lse, so = self.cache.attn(q.cuda(), dl, max_len=max_len, scores=torch.zeros(self.n, self.o.table.shape[1], device="cuda") if scores is None else scores,
                                       softmax_scale=scale, return_lse=True)
        self.check_attend(q, lens if expect is None else expect, out, lse, so, scores, scale)
        return out, lse, so

    def check_attend(self, q, lens, out, lse, so, scores=None, scale=0.0):
        res, mass = self.o.attend(q.double().numpy(), lens, scale or None)
        out, lse, so = (x.double().cpu().numpy() for x in (out, lse, so))
        before = 0.0 if scores is None else scores.double().cpu().numpy()
        for s, (ro, rl, spread, reach, n, vmax) in enumerate(res):
            # the query in fp16 behind a power of two: an element may lose 2^-25 of the head's largest, at most d of them
            # meet keys: the logit moves by less than d 2^-25 of the largest product, covered by doubling the logit's bound
            tol = po.out_tolerance(ro, spread, vmax, n, self.d, 2 * reach, HALF_STEP[self.dtype], 2.0 ** -11)
            err = np.abs(out[s] - ro)
            assert (err <= tol).all(), (s, n, float((err / tol).max()))
            if n == 0:
                assert np.isneginf(lse[s]).all()
            else:
                assert (np.abs(lse[s] - rl) <= po.lse_tolerance(rl, self.d, 2 * reach)).all(), s
            rel = 2 * po.logit_error(self.d, 2 * reach) + 2.0 ** -20
            want = mass[s] + (before if scores is None else before[s])
            assert (np.abs(so[s] - want) <= rel * mass[s] + 2.0 ** -22 * np.abs(want) + 1e-30).all(), (s, float(np.abs(so[s] - want).max()))


SHAPES = [
    (2, 128, 64, torch.bfloat16, "int8", 8), (4, 64, 16, torch.float16, "e4m3", 8), (1, 128, 128, torch.float16, "int8", 7),
    (2, 64, 32, torch.bfloat16, "e4m3", 2), (1, 128, 32, torch.bfloat16, "int8", 16), (2, 64, 128, torch.float16, "int8", 6),
    (1, 64, 16, torch.bfloat16, "int8", 12), (3, 128, 16, torch.float16, "e4m3", 3),
]  # KV heads, d, block, type, code, query heads


# ---- append -------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,block,dtype,code,hq", SHAPES)
def test_append_writes_what_the_quantizer_says(hkv, d, block, dtype, code, hq):
    p = Pair(5, 6, hkv, d, block, dtype, code, 3)
    for counts in ([block, 1, 0, 2 * block + 3, block - 1], [1, block - 1, 3, block, 1], [block + 2, 2 * block, 5, 1, 2 * block - 1], [0, 0, 1, 0, 0]):
        p.append(counts)
        p.check_state()
    for _ in range(3):
        p.append([1] * 5, single=True)
        p.check_state()
    assert int(p.cache.status) == 0


@pytest.mark.gpu
def test_append_codes_are_exact_for_awkward_values():
    # magnitudes over the whole range of the type, ties, zeros, values that are not finite
    p = Pair(8, 2, 1, 128, 32, torch.bfloat16, "int8", 5)
    g = torch.Generator().manual_seed(2)
    x = [torch.randn((32, 1, 128), generator=g) * s for s in (1e-38, 1e-30, 3e38 / 6, 1.0)]
    ties = torch.arange(32 * 128).reshape(32, 1, 128).float() % 255 - 127
    x += [ties * 0.5 + 0.0, torch.zeros(32, 1, 128), torch.randn((32, 1, 128), generator=g), torch.randn((32, 1, 128), generator=g)]
    x = torch.cat(x).clamp(-3.3e38, 3.3e38).to(torch.bfloat16)
    x[6 * 32 + 3, 0, 5] = float("nan")
    x[7 * 32 + 31, 0, 127] = float("-inf")
    for code in ("int8", "e4m3"):
        p = Pair(8, 2, 1, 128, 32, torch.bfloat16, code, 5)
        p.append([32] * 8, kv=[x, x.flip(0)])
        p.check_state()


@pytest.mark.gpu
def test_append_leaves_alone_what_it_should():
    p = Pair(4, 2, 2, 64, 16, torch.float16, "int8", 7)
    p.append([20, 3, 16, 31])
    p.append([5, 2, 1, 1], start=[-1, 3, 16, 31])  # the first sequence is padding
    p.check_state()
    assert p.lens.tolist() == [20, 5, 17, 32]
    p.append([4, 0, 40, 1], start=[20, 5, 17, 32])  # past the table: the third and fourth are cut
    p.check_state()
    assert int(p.cache.status) == 11


@pytest.mark.gpu
def test_append_to_absent_and_impossible_pages():
    p = Pair(3, 3, 2, 64, 16, torch.bfloat16, "int8", 7)
    p.o.table[0, 1] = -1
    p.cache.block_table.copy_(torch.from_numpy(p.o.table))
    p.append([40, 20, 48])
    p.check_state()
    assert int(p.cache.status) == 0
    p.o.table[1, 1], p.o.table[2, 0] = p.n_pages, -7
    p.cache.block_table.copy_(torch.from_numpy(p.o.table))
    p.append([0, 20, 0])
    p.check_state()
    assert int(p.cache.status) == 10
    p.attend(4)
    assert int(p.cache.status) == 10


@pytest.mark.gpu
def test_append_of_prompts_without_a_bound_keeps_every_token():
    p, r = (Pair(3, 4, 2, 64, 16, torch.float16, "int8", 27) for _ in range(2))
    k, v = p.random(60)
    p.append([33, 0, 27], kv=[k, v])
    dev = dict(dtype=torch.int32, device="cuda")
    r.cache.append(k.cuda(), v.cuda(), torch.zeros(3, **dev), torch.tensor([0, 33, 33, 60], **dev))
    r.o, r.lens = p.o, p.lens
    r.check_state()
    assert int(r.cache.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("cu,max_new,kept", [
    ([0, 10, 12], 7, [7, 2]),     # more tokens than the bound
    ([0, 3, 13], 10, [3, 0]),     # rows past the input
    ([-2, 3, 5], 10, [0, 2]),     # rows before it
    ([0, 6, 4], 10, [6, 0]),      # falling bounds
    ([0, 6, 4], 10, [0, 0]),      # the same for a sequence that is not to be touched: only the other one counts
])
def test_append_says_so_where_it_drops_rows(cu, max_new, kept):
    p = Pair(2, 2, 1, 64, 16, torch.float16, "int8", 29)
    k, v = p.random(12)
    start = np.array([0 if kept[0] else -1, 0])
    if cu[0] < 0:
        start[0] = 0
    p.o.append([x.double().numpy() for x in (k, v)], start, kept, [max(cu[0], 0), cu[1]])
    p.lens = np.where(start >= 0, kept, 0)
    dev = dict(dtype=torch.int32, device="cuda")
    p.cache.append(k.cuda(), v.cuda(), torch.tensor(start, **dev), torch.tensor(cu, **dev), max_new)
    p.check_state()
    for x in (p.cache.k_tail, p.cache.v_tail):  # nothing behind them either
        assert all(x[s, :, n:].isnan().all() for s, n in enumerate(kept))
    assert int(p.cache.status) == 11


@pytest.mark.gpu
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("code,dtype", [("int8", torch.bfloat16), ("e4m3", torch.float16)])
def test_append_says_so_where_a_block_is_not_finite(bad, code, dtype):
    p = Pair(2, 3, 2, 64, 16, dtype, code, 31)
    k, v = p.random(40)
    v[21, 1, 7] = float(bad)  # in the open block of the second sequence: kept as it is
    p.append([16, 15], kv=[k[:31], v[:31]])
    p.check_state()
    assert int(p.cache.status) == 0
    p.append([0, 1], kv=[k[31:32], v[31:32]])  # which is full now
    p.check_state()
    assert int(p.cache.status) == 13


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_codes_of_zeros_and_of_what_rounds_to_zero(code):
    # the same block at scales inside and outside the range in which quotients come from products
    dev = dict(dtype=torch.int32, device="cuda")
    x = torch.randn((16, 1, 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).float()
    x[0, 0, 0], x[3, 0, 5], x[4, 0, 6] = 5.0, -0.0, 0.0
    got = []
    for gain in (2.0 ** -70, 1.0, 2.0 ** 10, 2.0 ** 80):
        c = binding.Kv8Cache.allocate(1, 1, 1, 1, 64, 16, torch.bfloat16, CODES[code])
        c.block_table.zero_()
        y = (x * gain).to(torch.bfloat16)
        y[5, 0, 7], y[6, 0, 8] = -1e-39, 1e-39  # far below half a code at the larger scales, but not zeros
        c.append(y.cuda(), y.cuda(), torch.zeros(1, **dev), torch.tensor([0, 16], **dev))
        codes = c.k_codes.view(torch.uint8).cpu()[0, 0]
        assert codes[3, 5] == 0 and codes[4, 6] == 0
        got.append(codes)
    assert all(torch.equal(got[0], z) for z in got[1:])


@pytest.mark.gpu
def test_append_takes_strided_rows():
    hkv, d, dtype = 2, 128, torch.bfloat16
    p, r = (Pair(2, 4, hkv, d, 32, dtype, "e4m3", 9) for _ in range(2))
    k, v = p.random(70)
    p.append([33, 37], kv=[k, v])
    both = torch.stack([k, v], dim=1).cuda()  # one projection's output
    dev = dict(dtype=torch.int32, device="cuda")
    r.cache.append(both[:, 0], both[:, 1], torch.zeros(2, **dev), torch.tensor([0, 33, 70], **dev), 37)
    for name in ("k_codes", "v_codes", "k_tail", "v_tail"):
        assert torch.equal(getattr(p.cache, name).view(torch.uint8), getattr(r.cache, name).view(torch.uint8))


# ---- attention ------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,block,dtype,code,hq", SHAPES)
def test_attention_and_masses(hkv, d, block, dtype, code, hq):
    mb = max(4, 640 // block)
    p = Pair(6, mb, hkv, d, block, dtype, code, 1)
    cap = mb * block
    p.append([1, block, cap, block + 1, 0, cap // 2 - 1])
    scores = torch.rand((6, mb), generator=p.g).cuda()
    p.attend(hq, scores=scores)
    p.attend(hq, scale=0.2)
    p.attend(hq, gain=6.0)
    p.append([1, 1, 0, 1, 1, 1], start=[1, block, -1, block + 1, 0, cap // 2 - 1])
    p.attend(hq)
    assert int(p.cache.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,hkv,block,code", [(1, 8, 64, "int8"), (3, 2, 16, "e4m3"), (1, 1, 128, "int8"), (40, 4, 32, "int8")])
def test_long_and_many(n, hkv, block, code):
    longest = 9000 if n < 10 else 700
    mb = -(-longest // block) + 1
    p = Pair(n, mb, hkv, 128, block, torch.bfloat16, code, 2)
    rng = np.random.default_rng(0)
    counts = [longest] + [int(x) for x in rng.integers(0, longest, n - 1)]
    p.append(counts)
    p.attend(4 * hkv)
    p.attend(4 * hkv, max_len=longest)


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,hq,d,block,dtype,code", [(2, 4, 64, 32, torch.bfloat16, "int8"), (1, 16, 128, 128, torch.float16, "e4m3"), (2, 8, 128, 16, torch.float16, "int8")])
def test_long_contexts_lose_no_part(hkv, hq, d, block, dtype, code):
    # within what independent roundings leave, and that a sum without one in 256 of the keys is not
    n = 50000
    p = Pair(1, -(-n // block) + 1, hkv, d, block, dtype, code, 37)
    k, v = (torch.randn((n, hkv, d), generator=p.g).to(dtype) for _ in range(2))
    p.cache.append(k.cuda(), v.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    q = torch.randn((1, hq, d), generator=p.g).to(dtype)
    out = p.cache.attn(q.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda")).double().cpu().numpy()
    full, kv = n // block, []  # what the codes on the device stand for, and the open block
    pages = p.cache.block_table[0, :full].long()
    for codes, scale, x in ((p.cache.k_codes, p.cache.k_scale, k), (p.cache.v_codes, p.cache.v_scale, v)):
        y = (codes[pages].double() * scale[pages].double()[..., None, None]).transpose(1, 2).reshape(-1, hkv, d).cpu()
        assert (y - x[:full * block].double()).abs().max() < 0.2
        kv.append(torch.cat([y, x[full * block:].double()]).numpy())
    qn = q.double().numpy()
    ro, _, _, _ = po.attention(qn, *kv, False)
    vmax = float(np.abs(kv[1]).max())
    reach = 2 * d ** -0.5 * float(np.abs(qn).sum(-1).max()) * float(np.abs(kv[0]).max())  # codes enter with an offset: see the outliers' test
    tol = po.rms_tolerance(ro, *po.roundings(qn, *kv, False), d, reach, HALF_STEP[dtype], 2.0 ** -11, True) + 2 * 32 * 2.0 ** -24 * 2 * vmax
    rms = lambda x: float(np.sqrt(np.mean(x * x)))  # noqa: E731
    assert rms(out - ro) <= tol, rms(out - ro) / tol
    for i in (0, 100, 255):
        less = kv[1].copy()
        less[i * n // 256:(i + 1) * n // 256] = 0.0
        assert rms(po.attention(qn, kv[0], less, False)[0] - ro) > 3 * tol


@pytest.mark.gpu
def test_hundreds_of_sequences():
    p = Pair(300, 3, 1, 64, 16, torch.float16, "int8", 14)
    rng = np.random.default_rng(4)
    p.append([int(x) for x in rng.integers(0, 48, 300)])
    p.check_state()
    p.attend(2)
    p.append([1] * 300, single=True)
    p.attend(2)


@pytest.mark.gpu
def test_two_calls_at_once():
    p = Pair(3, 30, 2, 128, 32, torch.bfloat16, "e4m3", 15)
    p.append([900, 64, 333])
    q = torch.randn((3, 8, 128), generator=p.g).to(torch.bfloat16).cuda()
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (p.lens, [32, 0, 320])]
    scores = torch.zeros((3, 30), device="cuda")
    want = [p.cache.attn(q, x, scores=scores, return_lse=True) for x in lens]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[p.cache.attn(q, x, scores=scores, return_lse=True, stream=st) for x, st in zip(lens, streams)] for _ in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for pair in got for g, w in zip(pair, want) for a, b in zip(g, w))


@pytest.mark.gpu
def test_pages_shared_by_sequences_are_read_by_both():
    p = Pair(2, 6, 2, 64, 16, torch.float16, "int8", 16)
    p.append([40, 40])
    p.o.table[1, :2] = p.o.table[0, :2]  # a common prefix of two blocks
    p.cache.block_table.copy_(torch.from_numpy(p.o.table))
    p.attend(4)
    assert int(p.cache.status) == 0


@pytest.mark.gpu
def test_lengths_out_of_range_and_absent_blocks():
    p = Pair(5, 4, 2, 128, 32, torch.bfloat16, "int8", 4)
    p.append([128, 100, 64, 33, 128])
    p.o.table[0, 1] = p.o.table[4, 0] = p.o.table[4, 1] = p.o.table[4, 2] = p.o.table[4, 3] = -1
    p.cache.block_table.copy_(torch.from_numpy(p.o.table))
    p.attend(8)
    assert int(p.cache.status) == 0
    p.attend(8, lens=[-3, 100, 64, 0, 128], expect=[0, 100, 64, 0, 128])
    assert int(p.cache.status) == 0
    # beyond the bound: cut to whole blocks
    p.attend(8, lens=[128, 100, 64, 33, 128], max_len=70, expect=[64, 64, 64, 33, 64])
    assert int(p.cache.status) == 11
    p.attend(8, lens=[0, 0, 0, 0, 0])


@pytest.mark.gpu
def test_blocks_of_very_different_size_and_logits_that_climb():
    p = Pair(2, 12, 1, 64, 16, torch.float16, "int8", 6)
    k, v = p.random(2 * 190)
    up = torch.linspace(0.01, 4.0, 190)[:, None, None]
    k[:190], k[190:] = (k[:190] * up).half(), (k[190:] * up.flip(0)).half()
    v = (v * torch.cat([10.0 ** torch.linspace(-3, 3, 190), 10.0 ** torch.linspace(3, -3, 190)])[:, None, None]).half()
    p.append([190, 190], kv=[k, v])
    p.attend(4, gain=3.0)


@pytest.mark.gpu
@pytest.mark.parametrize("code,d", [("int8", 128), ("e4m3", 128), ("int8", 64)])
def test_outlier_channels(code, d):
    # four channels 30 times the others: the block's scale follows them.  int8 codes enter the products with an offset of half
    # their range, so a logit's float32 sum has terms of up to 2 |q_c| amax: its error is bounded by that sum, not by
    # sum |q_c| |k_c|, and the same holds for the output with the values' largest magnitude.
    p = Pair(2, 40, 2, d, 32, torch.bfloat16, code, 17)
    k, v = p.random(1700)
    for x in (k, v):
        x[:, :, [3, 17, 40, 63]] *= 30
    p.append([1200, 500], kv=[k, v])
    q = torch.randn((2, 8, d), generator=p.g).to(torch.bfloat16)
    lens = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    out, lse, so = (x.double().cpu().numpy() for x in p.cache.attn(q.cuda(), lens, scores=torch.zeros((2, 40), device="cuda"), return_lse=True))
    res, mass = p.o.attend(q.double().numpy(), p.lens)
    for s, (ro, rl, spread, _, n, vmax) in enumerate(res):
        kmax = float(k.double().abs().max())
        reach = 2 * d ** -0.5 * float(q[s].double().abs().sum(-1).max()) * kmax
        tol = po.out_tolerance(ro, spread, vmax, n, d, reach, 2.0 ** -8, 2.0 ** -11) + 2 * 32 * 2.0 ** -24 * 2 * vmax
        assert (np.abs(out[s] - ro) <= tol).all()
        assert (np.abs(lse[s] - rl) <= po.lse_tolerance(rl, d, reach)).all()
        assert (np.abs(so[s] - mass[s]) <= 2 * po.logit_error(d, reach) * mass[s] + 1e-30).all()
        # and far inside that bound, as independent roundings are
        assert np.abs(lse[s] - rl).max() < 2e-5 and (np.abs(so[s] - mass[s]) <= 1e-4 * mass[s]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,block,hq", [(1, 128, 32, 8), (2, 64, 16, 4), (1, 64, 64, 12)])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_blocks_near_the_end_of_the_types_range(hkv, d, block, hq, code):
    # |x| up to 1e34.  A running sum has at most 100 terms of at most 2^8 x 1e34: 2.6e38, a float32.
    p = Pair(2, 8, hkv, d, block, torch.bfloat16, code, 23)
    kv = [(1e34 * (2 * torch.rand((150, hkv, d), generator=p.g) - 1)).to(torch.bfloat16) for _ in range(2)]
    p.append([100, 50], kv=kv)
    p.check_state()
    p.attend(hq, gain=2e-34)  # logits of ordinary size
    # one key whose logits are near the end of float32, zeros beside it: all of the weight is on its token
    p = Pair(1, 8, hkv, d, block, torch.bfloat16, code, 24)
    k, v = torch.zeros((90, hkv, d)), torch.randn((90, hkv, d), generator=p.g)
    k[5, :, 3] = 1e34
    p.append([90], kv=[k.to(torch.bfloat16), v.to(torch.bfloat16)])
    q = torch.zeros((1, hq, d), dtype=torch.bfloat16)
    q[:, :, 3] = 1000
    out = p.cache.attn(q.cuda(), torch.tensor([90], dtype=torch.int32, device="cuda")).double().cpu()
    rows = torch.from_numpy(p.o.rows(0, 90)[1][5])  # [hkv, d], what the codes of token 5 stand for
    want = rows.repeat_interleave(hq // hkv, 0)[None]
    assert (out - want).abs().le(2.0 ** -8 * want.abs() + 2.0 ** -20).all()


@pytest.mark.gpu
def test_what_lies_behind_the_length_is_not_used():
    p = Pair(3, 4, 2, 64, 32, torch.float16, "e4m3", 8)
    p.append([40, 128, 97])
    for x in (p.cache.k_tail, p.cache.v_tail):
        x[0, :, 8:] = float("nan")
        x[1] = float("inf")
    p.cache.block_table[0, 1:] = 1 << 30  # an open block needs no page
    p.attend(2)
    assert int(p.cache.status) == 0
    # fewer tokens than were appended, at a block boundary
    p.attend(2, lens=[32, 96, 64])


@pytest.mark.gpu
def test_the_same_bits_every_time_and_in_a_graph_and_on_another_stream():
    p = Pair(4, 20, 4, 128, 64, torch.bfloat16, "int8", 11)
    p.append([1200, 5, 640, 77])
    q = torch.randn((4, 16, 128), generator=p.g).to(torch.bfloat16).cuda()
    lens = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    scores = torch.zeros((4, 20), device="cuda")
    want = p.cache.attn(q, lens, scores=scores, return_lse=True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, p.cache.attn(q, lens, scores=scores, return_lse=True)))
    assert torch.equal(p.cache.attn(q, lens), want[0])  # without masses
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = p.cache.attn(q, lens, scores=scores, return_lse=True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # a decode step in a graph: append, attend, masses in place, lengths advanced on the device
    k, v = (x.cuda() for x in p.random(4))
    out, acc, dev = torch.zeros_like(q), torch.zeros_like(scores), lens.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.cache.append(k, v, dev)
        dev.add_(1)
        p.cache.attn(q, dev, scores=acc, scores_out=acc, out=out)
    kv = [k.cpu(), v.cpu()]
    total = torch.zeros((4, 20), dtype=torch.float64)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        p.o.append([x.double().numpy() for x in kv], p.lens, [1] * 4, range(4))
        p.lens = p.lens + 1
        _, mass = p.o.attend(q.double().cpu().numpy(), p.lens)
        total += torch.from_numpy(mass)
    assert dev.tolist() == p.lens.tolist()
    p.check_state()
    assert (acc.double().cpu() - total).abs().max() < 1e-3
    _, lse, so = p.cache.attn(q, dev, scores=scores, return_lse=True)
    p.check_attend(q.cpu(), p.lens, out, lse, so)


@pytest.mark.gpu
def test_pools_beyond_32_bit_offsets():
    # 2^31 bytes of codes lie below the pages that are used
    hkv, d, block = 8, 128, 128
    n_pages = (1 << 31) // (hkv * d * block) + 40
    c = binding.Kv8Cache.allocate(n_pages, 1, 8, hkv, d, block, torch.float16, torch.int8)
    c.block_table[0] = torch.arange(n_pages - 8, n_pages, dtype=torch.int32)
    small = binding.Kv8Cache.allocate(8, 1, 8, hkv, d, block, torch.float16, torch.int8)
    small.block_table[0] = torch.arange(8, dtype=torch.int32)
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn((1000, hkv, d), generator=g).half().cuda() for _ in range(2))
    dev = dict(dtype=torch.int32, device="cuda")
    q = torch.randn((1, 32, d), generator=g).half().cuda()
    got = []
    for x in (c, small):
        x.append(k, v, torch.zeros(1, **dev), torch.tensor([0, 1000], **dev), 1000)
        got.append(x.attn(q, torch.tensor([1000], **dev)))
    assert torch.equal(got[0], got[1])
    assert torch.equal(c.k_codes[-8:-1], small.k_codes[:7]) and int(c.k_codes[0].abs().max()) == 0


@pytest.mark.gpu
def test_bindings_refuse_what_the_library_cannot_see():
    p = Pair(2, 4, 2, 64, 32, torch.float16, "int8")
    c = p.cache
    q, lens = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    k = torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
    for call in (lambda: c.attn(q.float(), lens), lambda: c.attn(q[:1], lens), lambda: c.attn(q, lens.long()), lambda: c.attn(q, lens, scores=torch.zeros(2, 3, device="cuda")),
                 lambda: c.attn(q.transpose(0, 1).contiguous().transpose(0, 1), lens), lambda: c.append(k, k.float(), lens), lambda: c.append(k[:, :1], k[:, :1], lens),
                 lambda: c.append(k, k, lens.cpu()), lambda: c.append(k, k.transpose(0, 1).contiguous().transpose(0, 1), lens),
                 lambda: binding.Kv8Cache(c.k_codes.float(), c.v_codes, c.k_scale, c.v_scale, c.k_tail, c.v_tail, c.block_table),
                 lambda: binding.Kv8Cache(c.k_codes, c.v_codes, c.k_scale[:3], c.v_scale, c.k_tail, c.v_tail, c.block_table),
                 lambda: binding.qevict_kv8_evict(c.block_table, lens, torch.zeros(2, 4, device="cuda").half(), 32, 10, 3),
                 lambda: binding.qevict_kv8_evict(c.block_table, lens, torch.zeros(2, 4, device="cuda"), 32, 10, 3, 2, 2)):
        with pytest.raises(binding.QEvictError):
            call()


@pytest.mark.gpu
def test_sizes_that_do_not_fit_their_fields_are_refused():
    p = Pair(2, 4, 2, 64, 32, torch.float16, "int8")
    p.append([40, 3])
    c = p.cache
    q, lens = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    k = torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
    cu, x = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), torch.zeros(2, 4, device="cuda")
    for call in (lambda: c.append(k, k, lens, cu, (1 << 32) + 1), lambda: c.append(k, k, lens, cu, 1.5), lambda: c.append(k, k, lens, cu, -(1 << 32) + 1),
                 lambda: c.attn(q, lens, max_len=(1 << 32) + 40), lambda: c.attn(q, lens, max_len="40"),
                 lambda: binding.qevict_kv8_evict(c.block_table, lens, x, 32, 10, (1 << 32) + 3), lambda: binding.qevict_prompt_attn(q, k, k, cu[:2], max_q=(1 << 32) + 2),
                 lambda: binding.qevict_prompt_attn(q, k, k, cu[:2], softmax_scale=1e39)):
        with pytest.raises(binding.QEvictError):
            call()
    p.check_state()  # nothing has been stored
    c.append(k, k, torch.full_like(lens, -1), cu, np.int64(1))
    assert torch.equal(c.attn(q, lens, max_len=np.int32(40)), c.attn(q, lens, max_len=40))


@pytest.mark.gpu
def test_a_stream_of_another_device_is_refused():
    class Elsewhere:  # what the check sees of a stream
        device, device_index, stream_id, device_type, cuda_stream = torch.device("cuda", 5), 5, 0, 1, 0

    p = Pair(2, 4, 2, 64, 32, torch.float16, "int8")
    c, at = p.cache, Elsewhere()
    q, lens = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    k = torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
    cu, x = torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.zeros(2, 4, device="cuda")
    for call in (lambda s: c.append(k, k, lens, stream=s), lambda s: c.attn(q, lens, stream=s), lambda s: binding.qevict_prompt_attn(q, k, k, cu, stream=s),
                 lambda s: binding.qevict_kv8_evict(c.block_table, lens, x, 32, 10, 3, stream=s)):
        with pytest.raises(binding.QEvictError, match="stream belongs to"):
            call(at)
        call(torch.cuda.Stream())
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_masses_alone_and_an_output_in_the_queries_place():
    p = Pair(2, 8, 2, 128, 32, torch.bfloat16, "int8", 41)
    p.append([200, 77])
    q = torch.randn((2, 8, 128), generator=p.g).to(torch.bfloat16).cuda()
    lens = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    want, so = p.cache.attn(q, lens, scores=torch.zeros((2, 8), device="cuda"))
    got, mass = p.cache.attn(q, lens, scores_out=torch.full((2, 8), 7.0, device="cuda"))  # without scores: from zero
    assert torch.equal(got, want) and torch.equal(mass, so)
    got = p.cache.attn(q, lens, out=q)
    assert got is q and torch.equal(got, want)


@pytest.mark.gpu
def test_empty_batches_and_a_bound_of_zero():
    c = binding.Kv8Cache.allocate(4, 0, 2, 2, 64, 16, torch.float16)
    i32 = dict(dtype=torch.int32, device="cuda")
    none = torch.zeros(0, **i32)
    c.append(torch.zeros((0, 2, 64), device="cuda").half(), torch.zeros((0, 2, 64), device="cuda").half(), none)
    assert c.attn(torch.zeros((0, 4, 64), device="cuda").half(), none).shape == (0, 4, 64)
    got = binding.qevict_kv8_evict(c.block_table, none, torch.zeros((0, 2), device="cuda"), 16, 4, 1)
    assert got["block_table"].shape == (0, 2)
    p = Pair(2, 4, 1, 64, 16, torch.float16, "e4m3", 43)
    p.append([40, 5])
    p.attend(2, max_len=0, expect=[0, 0], scores=torch.rand((2, 4)).cuda())
    assert int(p.cache.status) == 11


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,hq,d,block,dtype,code", [(300, 300, 64, 16, torch.float16, "int8"), (96, 768, 64, 32, torch.bfloat16, "e4m3"), (64, 1024, 64, 16, torch.bfloat16, "int8")])
def test_many_heads(hkv, hq, d, block, dtype, code):
    p = Pair(2, 4, hkv, d, block, dtype, code, 45)
    p.append([3 * block + 5, block - 1])
    p.check_state()
    p.attend(hq, scores=torch.rand((2, 4), generator=p.g).cuda())


@pytest.mark.gpu
def test_as_many_sequences_as_a_cache_takes():
    p = Pair(8192, 3, 1, 64, 16, torch.float16, "e4m3", 47)
    lens = np.random.default_rng(6).integers(0, 46, 8192)
    lens[[0, 8191]] = [0, 48]
    p.append([int(x) for x in lens])
    p.check_state()
    p.attend(2)
    assert int(p.cache.status) == 0


# ---- eviction ---------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("n_equal", [0, 16384, 9000])
def test_eviction_from_the_longest_tables(n_equal):
    x = torch.rand((2, 16384), generator=torch.Generator().manual_seed(49))
    x[:, :n_equal] = 0.25
    table, lens, x = _evict_case(2, 16384, 16, [16384 * 16, 16383 * 16 + 5], x, 2 * 16384, 49)
    want = oracle.evict(table.numpy(), lens.numpy(), x.numpy(), 16, 2 * 16384, 5000, 3, 70)
    _check_evict(binding.qevict_kv8_evict(table.cuda(), lens.cuda(), x.cuda(), 16, 2 * 16384, 5000, 3, 70), want)


def _evict_case(n, mb, block, lens, scores, n_pages, seed=0):
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(max(n * mb, 1), generator=g).int().view(n, mb)
    return table, torch.tensor(lens, dtype=torch.int32), scores.float()


def _check_evict(got, want):
    for name, x in want.items():
        y = got[name].cpu().numpy()
        assert np.array_equal(y, x, equal_nan=name == "scores"), name


@pytest.mark.gpu
@pytest.mark.parametrize("n,mb,block,budget,sink,recent", [(1, 8, 16, 4, 1, 1), (3, 1000, 32, 200, 2, 3), (2, 1025, 16, 1000, 0, 0), (4, 70, 64, 0, 0, 0), (3, 300, 16, 5, 2, 3), (2, 9000, 16, 2048, 1, 8)])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_eviction_keeps_the_best(n, mb, block, budget, sink, recent, kind):
    g = torch.Generator().manual_seed(mb)
    x = torch.exp(2 * torch.randn((n, mb), generator=g))
    if kind == "ties":
        x = torch.round(torch.rand((n, mb), generator=g) * 3)
    if kind == "odd":  # signs, zeros of both, infinities, not-a-numbers
        x = x * torch.sign(torch.randn((n, mb), generator=g))
        pick = torch.randint(0, 9, (n, mb), generator=g)
        for i, v in enumerate((0.0, -0.0, float("inf"), float("-inf"), float("nan"))):
            x[pick == i] = v
    lens = [mb * block - 1 - (i * block * mb) // 7 for i in range(n)]
    lens[-1] = mb * block if n > 1 else lens[-1]
    table, lens, x = _evict_case(n, mb, block, lens, x, n * mb, 1)
    n_pages = n * mb - 3  # a few ids lie outside the pool
    want = oracle.evict(table.numpy(), lens.numpy(), x.numpy(), block, n_pages, budget, sink, recent)
    got = binding.qevict_kv8_evict(table.cuda(), lens.cuda(), x.cuda(), block, n_pages, budget, sink, recent)
    _check_evict(got, want)
    t, l, s = table.cuda(), lens.cuda(), x.cuda()
    got = binding.qevict_kv8_evict(t, l, s, block, n_pages, budget, sink, recent, in_place=True)
    assert got["block_table"] is t and got["lens"] is l and got["scores"] is s
    _check_evict(got, want)


@pytest.mark.gpu
def test_eviction_of_sequences_that_need_none():
    table, lens, x = _evict_case(5, 40, 16, [-1, 0, 15, 16 * 7, 16 * 8 + 3], torch.rand(5, 40), 200)
    want = oracle.evict(table.numpy(), lens.numpy(), x.numpy(), 16, 200, 8, 1, 2)
    got = binding.qevict_kv8_evict(table.cuda(), lens.cuda(), x.cuda(), 16, 200, 8, 1, 2)
    _check_evict(got, want)
    assert got["n_freed"].tolist() == [0] * 5 and torch.equal(got["block_table"].cpu(), table)


# ---- together ----------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,code,block", [(torch.bfloat16, "int8", 32), (torch.float16, "e4m3", 16)])
def test_prompt_then_decode_under_a_budget(dtype, code, block):
    """Prompt attention, append of the prompt, decode steps with masses, eviction, more steps in the freed pages."""
    hkv, hq, d, n, mb = 2, 8, 64, 3, 24
    p = Pair(n, mb, hkv, d, block, dtype, code, 13)
    prompts = [10 * block + 5, 3, 8 * block]
    k, v = p.random(sum(prompts))
    q = torch.randn((sum(prompts), hq, d), generator=p.g).to(dtype)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32, device="cuda")
    out, lse = binding.qevict_prompt_attn(q.cuda(), k.cuda(), v.cuda(), cu, max_q=max(prompts), max_k=max(prompts), return_lse=True)
    a = 0
    for m in prompts:
        ro, rl, spread, reach = po.attention(q[a:a + m].double().numpy(), k[a:a + m].double().numpy(), v[a:a + m].double().numpy())
        u = HALF_STEP[dtype]
        vmax = float(v[a:a + m].double().abs().max())
        assert (np.abs(out[a:a + m].double().cpu().numpy() - ro) <= po.out_tolerance(ro, spread, vmax, m, d, reach, u, u)).all()
        a += m
    p.append(prompts, kv=[k, v])
    scores = torch.zeros((n, mb), device="cuda")
    free = []
    for step in range(2 * block + 3):
        p.append([1] * n, single=True)
        _, _, scores = p.attend(hq, scores=scores)
        if step % block == block - 1:
            lens = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
            want = oracle.evict(p.o.table, p.lens, scores.cpu().numpy(), block, p.n_pages, 6, 1, 2)
            got = binding.qevict_kv8_evict(p.cache.block_table, lens, scores, block, p.n_pages, 6, 1, 2, in_place=True)
            _check_evict(got, want)
            # freed pages go to the end of the tables that lost them
            for s in range(n):
                m = int(want["n_freed"][s])
                if m:
                    row = want["block_table"][s]
                    at = int((row >= 0).sum())
                    row[at:at + m] = want["freed"][s, :m]
                    free += want["freed"][s, :m].tolist()
            p.o.table = want["block_table"]
            p.cache.block_table.copy_(torch.from_numpy(p.o.table))
            p.lens = want["lens"].astype(np.int64)
    p.check_state()
    assert len(free) > 0 and int(p.cache.status) == 0
