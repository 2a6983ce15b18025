"""The 16-bit paged cache against a float64 evaluation: append with the rotation, attention of new tokens over the pages."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import prompt, rotary as oracle
from paper_2608_05326_b200 import binding

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


# ---- refusals: checked before anything reaches a device --------------------------------------------------------
def _fill(a, values):
    for n, x in values.items():
        field = getattr(a, n)
        if isinstance(field, C.Array):
            for i, y in enumerate(x):
                field[i] = y
        else:
            setattr(a, n, x)
    return a


def _view(**over):
    c = binding.qevict_kv16_cache()
    values = dict(struct_size=C.sizeof(c), device=0, dtype=1, n_seqs=2, n_kv_heads=2, head_dim=64, block=16, max_blocks=4, n_pages=8, reserved=0,
                  k_pages=4096, v_pages=4096, k_stride=(2048, 1024, 64), v_stride=(2048, 1024, 64), block_table=4096)
    values.update(over)
    return _fill(c, values)


VIEWS = [
    (dict(struct_size=8), 1, "struct_size"), (dict(device=-1), 1, "device"), (dict(dtype=2), 1, "dtype"), (dict(reserved=2), 1, "reserved"),
    (dict(n_seqs=-1), 1, "n_seqs"), (dict(n_kv_heads=0), 1, "n_kv_heads"), (dict(max_blocks=0), 1, "max_blocks"), (dict(n_pages=0), 1, "n_pages"),
    (dict(head_dim=96), 4, "head_dim"), (dict(block=48), 4, "block"), (dict(block=8), 4, "block"), (dict(n_kv_heads=2000), 4, "KV heads"), (dict(n_seqs=70000), 4, "sequences"),
    (dict(max_blocks=1 << 28), 4, "tokens"), (dict(k_pages=None), 1, "NULL"), (dict(block_table=None), 1, "NULL"), (dict(v_pages=4104), 1, "aligned"),
    (dict(status=4098), 1, "aligned"), (dict(k_stride=(2048, 1020, 64)), 1, "strides"), (dict(v_stride=(0, 1024, 64)), 1, "strides"), (dict(k_stride=(1 << 38, 1024, 64)), 1, "strides"),
]


def _append_args(view, **over):
    a = binding.qevict_kv16_append_args()
    values = dict(struct_size=C.sizeof(a), n_q_heads=4, cache=C.addressof(view), total_new=2, start=4096, k=4096, v=4096, q=4096, q_out=8192,
                  k_stride=(128, 64), v_stride=(128, 64), q_stride=(256, 64), q_out_stride=(256, 64))
    values.update(over)
    return _fill(a, values)


def _refused(call, status, word):
    with pytest.raises(binding.QEvictError) as e:
        binding._check(call)
    assert e.value.status == status and word in str(e.value), str(e.value)


@pytest.mark.parametrize("over,status,word", VIEWS)
def test_append_refuses_unusable_views(over, status, word):
    view = _view(**over)
    _refused(binding.lib().qevict_kv16_append(C.byref(_append_args(view)), None), status, word)


@pytest.mark.parametrize("over,status,word", [
    (dict(struct_size=8), 1, "struct_size"), (dict(cache=None), 1, "cache is NULL"), (dict(total_new=-1), 1, "total_new"), (dict(n_q_heads=-1), 1, "n_q_heads"),
    (dict(n_q_heads=1025), 4, "heads"), (dict(total_new=2 ** 31), 4, "tokens"), (dict(positions=4096), 1, "without a rotation"), (dict(total_new=1), 1, "at least n_seqs"),
    (dict(k=None), 1, "NULL"), (dict(v=None), 1, "NULL"), (dict(q=None), 1, "NULL"), (dict(q_out=None), 1, "NULL"), (dict(start=None), 1, "start"), (dict(start=4098), 1, "aligned"),
    (dict(cu_new=4098), 1, "aligned"), (dict(k=4104), 1, "aligned"), (dict(v_stride=(120, 60)), 1, "strides"), (dict(q_out=4096, q_out_stride=(512, 64)), 1, "its strides"),
])
def test_append_refuses_unusable_arguments(over, status, word):
    view = _view()
    _refused(binding.lib().qevict_kv16_append(C.byref(_append_args(view, **over)), None), status, word)


def test_append_of_nothing_needs_no_device():
    lib, empty, view = binding.lib(), _view(n_seqs=0, block_table=None), _view()
    assert lib.qevict_kv16_append(C.byref(_append_args(empty)), None) == 0
    assert lib.qevict_kv16_append(C.byref(_append_args(view, total_new=0, k=None, v=None, q=None, cu_new=4096)), None) == 0
    wide = binding.Rotation.standard(128)
    _refused(lib.qevict_kv16_append(C.byref(_append_args(view, rotation=wide._address)), None), 1, "more channels")


# ---- append ----------------------------------------------------------------------------------------------------
def _np(x):
    return x.double().cpu().numpy()


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _cu(lens, first=0):
    return _i32(np.concatenate([[first], first + np.cumsum(lens)]))


def _cache(lens, hkv, d, block, dtype, seed, extra=2, fill=None, by_token=False, table=None):
    """A cache with pages in a shuffled order for sequences of these lengths; by_token: pages [page, token, head, channel]."""
    g = torch.Generator().manual_seed(seed)
    need = [max(1, -(-n // block)) for n in lens]
    n_pages = sum(need) + extra
    perm = torch.randperm(n_pages, generator=g).to(torch.int32)
    if table is None:
        table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
        at = 0
        for s, m in enumerate(need):
            table[s, :m] = perm[at:at + m]
            at += m
    shape = (n_pages, block, hkv, d) if by_token else (n_pages, hkv, block, d)
    pools = []
    for _ in range(2):
        x = torch.randn(shape, generator=g).to(dtype) if fill is None else torch.full(shape, fill, dtype=dtype)
        pools.append(x.cuda().transpose(1, 2) if by_token else x.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    return binding.Kv16Cache(pools[0], pools[1], table.cuda(), status), pools, table.numpy(), status


def _rows(total, heads, d, dtype, seed):
    return torch.randn((total, heads, d), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _spec(n_pairs, n_axes=1, interleaved=False):
    freq, axes = 500000.0 ** (-np.arange(n_pairs) / n_pairs), list(np.arange(n_pairs) % n_axes)
    return binding.Rotation(freq, axes=axes, interleaved=interleaved), dict(inv_freq=freq, axes=axes, interleaved=interleaved)


def _close(got, want, size, pos, spec, dtype):
    tol = oracle.rotate_tolerance(want, size, pos, spec["inv_freq"], HALF_STEP[dtype], SMALLEST[dtype])
    err = np.abs(_np(got) - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


def _check_append(cache, pools, table, before, k, v, start, counts, first, rotated_k, k_tol):
    """Pages after the call: new rows where they belong, everything else with its bits."""
    want = oracle.Pages([_np(before[0]), _np(before[1])], table)
    tol = oracle.Pages([np.zeros(before[0].shape), np.zeros(before[0].shape)], table)
    want.append((rotated_k, _np(v)), start, counts, first)
    tol.append((k_tol, np.zeros(v.shape)), start, counts, first)
    for w in range(2):
        err = np.abs(_np(pools[w]) - want.pools[w])
        assert (err <= tol.pools[w]).all(), (w, float(err.max()))


APPENDS = [
    ([0], [1]), ([0], [16]), ([5], [77]), ([15], [1]), ([16], [17]), ([0, 31, 100, 7], [40, 1, 0, 130]), ([3, 64, 0], [1, 1, 1]), ([500], [300]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("start,counts", APPENDS)
@pytest.mark.parametrize("dtype,hq,hkv,d,block,n_pairs,interleaved,n_axes,by_token", [
    (torch.bfloat16, 32, 8, 128, 64, 64, False, 1, False), (torch.float16, 7, 1, 64, 16, 32, False, 3, True), (torch.bfloat16, 4, 2, 64, 32, 12, True, 2, False),
    (torch.float16, 0, 4, 128, 128, 32, True, 1, True), (torch.bfloat16, 3, 3, 128, 16, 0, False, 1, False),
])
def test_append(start, counts, dtype, hq, hkv, d, block, n_pairs, interleaved, n_axes, by_token):
    total = sum(counts)
    cache, pools, table, status = _cache([a + b for a, b in zip(start, counts)], hkv, d, block, dtype, 3, by_token=by_token)
    before = [x.clone() for x in pools]
    k, v = _rows(total, hkv, d, dtype, 1), _rows(total, hkv, d, dtype, 2)
    q = _rows(total, hq, d, dtype, 4) if hq else None
    first = np.concatenate([[0], np.cumsum(counts)])[:-1]
    place = np.concatenate([np.arange(a, a + b) for a, b in zip(start, counts)])[None]
    args = {}
    if n_pairs:
        rotation, spec = _spec(n_pairs, n_axes, interleaved)
        pos = place.repeat(n_axes, 0) if n_axes != 2 else np.random.default_rng(5).integers(0, 99999, (2, total))
        args = dict(rotation=rotation, positions=None if n_axes != 2 else _i32(pos))
        rk, size = oracle.rotate(_np(k), pos, **spec)
        ktol = oracle.rotate_tolerance(rk, size, pos, spec["inv_freq"], HALF_STEP[dtype], SMALLEST[dtype])
    else:
        rk, ktol = _np(k), np.zeros(k.shape)
    calls = [dict(cu_new=_cu(counts))] + ([dict()] if all(c == 1 for c in counts) else [])
    for how in calls:
        for x, y in zip(pools, before):
            x.copy_(y)
        got = cache.append(k, v, _i32(start), q=q, **how, **args)
        _check_append(cache, pools, table, before, k, v, start, counts, first, rk, ktol)
        if q is None:
            assert got is None
        elif n_pairs:
            rq, size = oracle.rotate(_np(q), pos, **spec)
            _close(got, rq, size, pos, spec, dtype)
        else:
            assert torch.equal(got, q)
    assert int(status) == 0


@pytest.mark.gpu
def test_what_the_rotation_gives_is_what_is_appended():
    # the same bits as the rotation by itself, whatever the number of tokens, and queries may be rotated in place
    hq, hkv, d, dtype = 28, 4, 128, torch.bfloat16
    rotation, _ = _spec(64, 3)
    for total in (1, 9, 5000):
        cache, pools, table, _ = _cache([total], hkv, d, 64, dtype, 6)
        qkv = _rows(total, hq + 2 * hkv, d, dtype, 7)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        pos = _i32(np.random.default_rng(8).integers(0, 99999, (3, total)))
        rq, rk = binding.qevict_rope(q, pos, rotation, k=k)
        same_k, same_v = k.clone(), v.clone()
        got = cache.append(k, v, _i32([0]), cu_new=_cu([total]), rotation=rotation, positions=pos, q=q, q_out=q)
        assert got is q and torch.equal(q, rq) and torch.equal(k, same_k) and torch.equal(v, same_v)
        rows = [x[torch.tensor(table[0], device="cuda").long()].transpose(1, 2).reshape(-1, hkv, d)[:total] for x in pools]
        assert torch.equal(rows[0], rk) and torch.equal(rows[1], v)


@pytest.mark.gpu
def test_what_cannot_be_stored_is_said_and_nothing_else_is_touched():
    hq, hkv, d, block, dtype = 2, 2, 64, 16, torch.float16
    rotation, spec = _spec(32)

    def call(start, cu, total, table=None, mb=4, code=0, stored=(), q_rows=None):
        n = len(start)
        t = torch.arange(n * mb, dtype=torch.int32).view(n, mb) if table is None else torch.tensor(table, dtype=torch.int32)
        cache, pools, tb, status = _cache([mb * block] * n, hkv, d, block, dtype, 9, fill=3.0, table=t)
        q, k, v = (_rows(total, h, d, dtype, 10 + i) for i, h in enumerate((hq, hkv, hkv)))
        out = torch.full_like(q, 7.0)
        cache.append(k, v, _i32(start), cu_new=None if cu is None else _i32(cu), rotation=rotation, q=q, q_out=out)
        assert int(status) == code, int(status)
        want = [np.full(x.shape, 3.0) for x in pools]
        tol = [np.zeros(x.shape) for x in pools]
        wq, tq = np.full(q.shape, 7.0), np.zeros(q.shape)
        for s, place, row in stored:
            rk, size = oracle.rotate(_np(k[row:row + 1]), [[place]], **spec)
            page = int(tb[s, place // block])
            want[0][page, :, place % block], want[1][page, :, place % block] = rk[0], _np(v[row])
            tol[0][page, :, place % block] = oracle.rotate_tolerance(rk, size, [[place]], spec["inv_freq"], HALF_STEP[dtype], SMALLEST[dtype])[0]
        for row, place in ([(r, p) for _, p, r in stored] if q_rows is None else q_rows):
            rq, size = oracle.rotate(_np(q[row:row + 1]), [[place]], **spec)
            wq[row], tq[row] = rq[0], oracle.rotate_tolerance(rq, size, [[place]], spec["inv_freq"], HALF_STEP[dtype], SMALLEST[dtype])[0]
        for got, w, t in ((pools[0], want[0], tol[0]), (pools[1], want[1], tol[1]), (out, wq, tq)):
            assert (np.abs(_np(got) - w) <= t).all()

    seq = lambda s, place, row, m: [(s, place + i, row + i) for i in range(m)]  # noqa: E731
    call([0, 5], [2, 6, 9], 12, stored=seq(0, 0, 2, 4) + seq(1, 5, 6, 3))                                 # rows before and behind the sequences
    call([-1, 5], [0, 6, 9], 9, stored=seq(1, 5, 6, 3))                                                   # left as it is
    call([0, 60], [0, 1, 9], 9, code=11, stored=seq(0, 0, 0, 1) + seq(1, 60, 1, 4), q_rows=[(0, 0)] + [(1 + i, 60 + i) for i in range(8)])
    call([0, 2 ** 31 - 1], [0, 1, 3], 3, code=11, stored=seq(0, 0, 0, 1), q_rows=[(0, 0), (1, 2 ** 31 - 1), (2, 2 ** 31)])
    call([0, 3], [0, 6, 2], 9, code=11, stored=seq(0, 0, 0, 6))                                           # falling bounds
    call([0, 3], [0, 6, 10], 9, code=11, stored=seq(0, 0, 0, 6))                                          # beyond the rows
    call([4, 3], [-2, 6, 9], 9, code=11, stored=seq(1, 3, 6, 3))                                          # before the rows
    call([0, 3], None, 4, stored=[(0, 0, 0), (1, 3, 1)])                                                  # one each; rows of nobody behind
    call([0, 3], [0, 20, 24], 24, table=[[1, -1], [2, 0]], mb=2, stored=seq(0, 0, 0, 16) + seq(1, 3, 20, 4), q_rows=[(i, i) for i in range(20)] + [(20 + i, 3 + i) for i in range(4)])
    for wrong in (-2, 6, 2 ** 31 - 1):
        call([0, 3], [0, 20, 24], 24, table=[[1, wrong], [2, 0]], mb=2, code=10, stored=seq(0, 0, 0, 16) + seq(1, 3, 20, 4), q_rows=[(i, i) for i in range(20)] + [(20 + i, 3 + i) for i in range(4)])


@pytest.mark.gpu
@pytest.mark.parametrize("n_seqs", [33, 1000, 5000])
def test_append_to_many_sequences(n_seqs):
    hkv, d, block, dtype = 1, 64, 16, torch.bfloat16
    rng = np.random.default_rng(n_seqs)
    counts, start = rng.integers(0, 4, n_seqs), rng.integers(0, 40, n_seqs)
    counts[-3:] = [0, 5, 0]
    cache, pools, table, status = _cache(list(start + counts), hkv, d, block, dtype, 11)
    before = [x.clone() for x in pools]
    k, v = _rows(int(counts.sum()), hkv, d, dtype, 12), _rows(int(counts.sum()), hkv, d, dtype, 13)
    cache.append(k, v, _i32(start), cu_new=_cu(counts))
    _check_append(cache, pools, table, before, k, v, start, counts, np.concatenate([[0], np.cumsum(counts)])[:-1], _np(k), np.zeros(k.shape))
    assert int(status) == 0


@pytest.mark.gpu
def test_append_past_2_to_the_31_elements():
    hkv, d, block, dtype = 8, 128, 128, torch.float16
    n_pages = (1 << 31) // (hkv * d * block) + 40
    pools = [torch.zeros((n_pages, hkv, block, d), dtype=dtype, device="cuda") for _ in range(2)]
    table = torch.tensor([[n_pages - 1, 0, n_pages - 30]], dtype=torch.int32, device="cuda")
    cache = binding.Kv16Cache(pools[0], pools[1], table)
    k, v = _rows(300, hkv, d, dtype, 14), _rows(300, hkv, d, dtype, 15)
    cache.append(k, v, _i32([0]), cu_new=_cu([300]))
    for x, y in zip(pools, (k, v)):
        rows = x[table[0].long()].transpose(1, 2).reshape(-1, hkv, d)
        assert torch.equal(rows[:300], y) and not rows[300:].any() and int((x != 0).any(-1).sum()) == 300 * hkv


@pytest.mark.gpu
def test_append_captured_with_the_lengths_advanced_inside():
    hq, hkv, d, block, dtype, n = 4, 2, 128, 16, torch.bfloat16, 3
    rotation, spec = _spec(64)
    cache, pools, table, _ = _cache([64] * n, hkv, d, block, dtype, 16, fill=0.0)
    q, k, v = (_rows(n, h, d, dtype, 17 + i) for i, h in enumerate((hq, hkv, hkv)))
    lens = _i32([0, 14, 30])
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(k, v, lens, rotation=rotation, q=q, q_out=out)
        lens += 1
    for step in range(4):
        k.copy_(_rows(n, hkv, d, dtype, 30 + step))
        graph.replay()
        pos = np.array([[step, 14 + step, 30 + step]])
        rq, size = oracle.rotate(_np(q), pos, **spec)
        _close(out, rq, size, pos, spec, dtype)
        rk, size = oracle.rotate(_np(k), pos, **spec)
        stored = torch.stack([pools[0][int(table[s, p // block]), :, p % block] for s, p in enumerate(pos[0])])
        _close(stored, rk, size, pos, spec, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = cache.append(k, v, lens, rotation=rotation, q=q, stream=side)
    side.synchronize()
    pos = np.array([[4, 18, 34]])
    rq, size = oracle.rotate(_np(q), pos, **spec)
    _close(got, rq, size, pos, spec, dtype)


@pytest.mark.gpu
def test_views_and_appends_of_the_binding_refuse_what_the_library_cannot_see():
    cache = binding.Kv16Cache.allocate(4, 2, 2, 2, 64, 16, torch.float16)
    kp, vp, t = cache.k_pages, cache.v_pages, cache.block_table
    rotation, _ = _spec(32)
    k, q, start = _rows(2, 2, 64, torch.float16, 1), _rows(2, 4, 64, torch.float16, 2), _i32([0, 0])
    for bad in (lambda: binding.Kv16Cache(kp.cpu(), vp, t), lambda: binding.Kv16Cache(kp.float(), vp.float(), t), lambda: binding.Kv16Cache(kp, vp[:3], t),
                lambda: binding.Kv16Cache(kp, vp.bfloat16(), t), lambda: binding.Kv16Cache(kp[0], vp[0], t), lambda: binding.Kv16Cache(kp, vp, t.long()),
                lambda: binding.Kv16Cache(kp, vp, t[:, :1]), lambda: binding.Kv16Cache(kp.transpose(2, 3), vp.transpose(2, 3), t), lambda: binding.Kv16Cache(kp, vp, t, start),
                lambda: cache.append(k.float(), k, start), lambda: cache.append(k, k[:1], start), lambda: cache.append(k[:, :1], k, start), lambda: cache.append(k, k, start[:1]),
                lambda: cache.append(k, k, start.long()), lambda: cache.append(k, k, start, cu_new=start), lambda: cache.append(k, k, start, q=q[:1]),
                lambda: cache.append(k, k, start, q_out=q), lambda: cache.append(k, k, start, q=q, q_out=q[:, :2]), lambda: cache.append(k, k, start, rotation=3),
                lambda: cache.append(k, k, start, positions=start), lambda: cache.append(k, k, start, rotation=rotation, positions=start.long()),
                lambda: cache.append(k[..., :32], k[..., :32], start)):
        with pytest.raises(binding.QEvictError):
            bad()


# ---- attention -------------------------------------------------------------------------------------------------
def _attn_args(view, **over):
    a = binding.qevict_kv16_attn_args()
    values = dict(struct_size=C.sizeof(a), n_q_heads=4, max_q=1, max_len=64, causal=1, softmax_scale=0.0, total_q=2, cache=C.addressof(view), lens=4096,
                  q=4096, out=8192, q_stride=(256, 64), out_stride=(256, 64))
    values.update(over)
    return _fill(a, values)


@pytest.mark.parametrize("over,status,word", VIEWS)
def test_attention_refuses_unusable_views(over, status, word):
    view, need = _view(**over), C.c_uint64()
    _refused(binding.lib().qevict_kv16_attn(C.byref(_attn_args(view)), None, 0, None), status, word)
    _refused(binding.lib().qevict_kv16_attn_scratch_bytes(C.byref(_attn_args(view)), C.byref(need)), status, word)


@pytest.mark.parametrize("over,status,word", [
    (dict(struct_size=8), 1, "struct_size"), (dict(cache=None), 1, "cache is NULL"), (dict(causal=2), 1, "causal"), (dict(max_q=-1), 1, "sizes"), (dict(max_len=-1), 1, "sizes"),
    (dict(total_q=-1), 1, "sizes"), (dict(n_q_heads=3), 1, "multiple"), (dict(n_q_heads=0), 1, "multiple"), (dict(softmax_scale=-1.0), 1, "softmax_scale"),
    (dict(softmax_scale=float("nan")), 1, "softmax_scale"), (dict(softmax_scale=3e38), 1, "softmax_scale"), (dict(max_q=2), 1, "without cu_q"), (dict(total_q=1), 1, "without cu_q"),
    (dict(n_q_heads=2048), 4, "heads"), (dict(total_q=2 ** 31), 4, "tokens"), (dict(q=None), 1, "NULL"), (dict(out=None), 1, "NULL"), (dict(lens=None), 1, "NULL"),
    (dict(q=4104), 1, "aligned"), (dict(lse=4098), 1, "aligned"), (dict(cu_q=4098), 1, "aligned"), (dict(q_stride=(250, 64)), 1, "strides"), (dict(out_stride=(256, 0)), 1, "strides"),
])
def test_attention_refuses_unusable_arguments(over, status, word):
    view = _view()
    _refused(binding.lib().qevict_kv16_attn(C.byref(_attn_args(view, **over)), None, 0, None), status, word)


def test_attention_scratch_and_nothing_to_do():
    lib, need, view = binding.lib(), C.c_uint64(1), _view(max_blocks=4096)
    for over in (dict(total_q=0, cu_q=4096), dict(max_q=0)):
        assert lib.qevict_kv16_attn(C.byref(_attn_args(view, **over)), None, 0, None) == 0
    assert lib.qevict_kv16_attn(C.byref(_attn_args(_view(n_seqs=0, block_table=None))), None, 0, None) == 0
    binding._check(lib.qevict_kv16_attn_scratch_bytes(C.byref(_attn_args(view, max_len=128)), C.byref(need)))
    assert need.value == 0  # one tile of keys has no parts
    long = _attn_args(view, max_len=65536)
    binding._check(lib.qevict_kv16_attn_scratch_bytes(C.byref(long), C.byref(need)))
    assert need.value > 0
    assert lib.qevict_kv16_attn(C.byref(long), None, 0, None) == 3 and b"scratch" in lib.qevict_last_error(None)
    assert lib.qevict_kv16_attn(C.byref(long), 4104, need.value, None) == 1 and b"aligned" in lib.qevict_last_error(None)
    assert lib.qevict_kv16_attn_scratch_bytes(C.byref(long), None) == 1


def _poison(pools, table, lens, block):
    """Not-a-number wherever no token is: behind the lengths, in pages of nobody."""
    pages = oracle.Pages([np.zeros((pools[0].shape[0], 1, block, 1))] * 2, table)
    used = np.zeros((pools[0].shape[0], block), bool)
    for s, n in enumerate(lens):
        for b in range(-(-n // block)):
            at = pages.place(s, b * block)
            if at is not None:
                used[at[0], :min(block, n - b * block)] = True
    hide = torch.tensor(~used, device="cuda")[:, None, :, None]
    for w, x in enumerate(pools):
        x.masked_fill_(hide, float("nan") if w else float("inf"))


def _check_seq(out, lse, q, k, v, n, places, causal, dtype, what, scale=None):
    """out [nq, Hq, d], lse [Hq, nq] of one sequence of n tokens, of which `places` are there."""
    ro, rl, spread, reach = prompt.attention(_np(q), k, v, causal, scale, places, n)
    vmax = float(np.abs(v).max()) if v.size else 0.0
    u = HALF_STEP[dtype]
    tol = prompt.out_tolerance(ro, spread, vmax, k.shape[0], q.shape[-1], reach, u, u)
    err = np.abs(_np(out) - ro)
    assert (err <= tol).all(), (what, float((err / tol).max()), float(err.max()))
    got, ok = _np(lse), np.isfinite(rl)
    assert (np.isneginf(got) == np.isneginf(rl)).all(), what
    assert (np.abs(got[ok] - rl[ok]) <= prompt.lse_tolerance(rl[ok], q.shape[-1], reach)).all(), what


def _check_attn(out, lse, q, pools, table, lens, nq, causal, dtype, q_first=0, scale=None, only=None):
    # (the pages as stored: what no token uses is not looked at)
    pages, at = oracle.Pages([_np(x) for x in pools], table), q_first
    for s, (m, n) in enumerate(zip(nq, lens)):
        if only is None or s in only:
            k, v, places = pages.rows(s, n)
            _check_seq(out[at:at + m], lse[:, at:at + m], q[at:at + m], k, v, n, places, causal, dtype, "sequence %d (%d of %d)" % (s, m, n), scale)
        at += m


def _case(nq, lens, hq, hkv, d, block, dtype, seed, by_token=False, gain=1.0, extra=2, mb=None):
    cache, pools, table, status = _cache(lens, hkv, d, block, dtype, seed, extra=extra, by_token=by_token)
    if mb is not None:  # a wider table, with page ids behind the lengths that nothing may use
        wide = torch.full((len(lens), mb), 1 << 30, dtype=torch.int32)
        for s, n in enumerate(lens):
            m = -(-n // block)
            wide[s, :m] = torch.tensor(table[s, :m])
        cache, table = binding.Kv16Cache(pools[0], pools[1], wide.cuda(), status), wide.numpy()
    _poison(pools, table, lens, block)
    return cache, pools, table, status, (_rows(sum(nq), hq, d, dtype, seed + 1) * gain).to(dtype)


LENS = [
    ([1], [1]), ([1], [128]), ([1], [129]), ([5], [5]), ([77], [77]), ([1], [300]), ([4], [1000]), ([33], [257]), ([300], [300]), ([129], [700]), ([260], [1500]),
    ([5, 0, 130, 1, 255], [5, 64, 130, 0, 600]), ([1, 1, 1], [1, 640, 129]), ([3, 200], [131, 456]), ([130, 4], [2, 3]), ([3, 2], [0, 2]),
]
LAYOUTS = [
    (torch.bfloat16, 32, 8, 128, 64, False), (torch.float16, 7, 1, 64, 16, True), (torch.bfloat16, 2, 2, 64, 128, False), (torch.float16, 28, 4, 128, 32, True),
    (torch.bfloat16, 16, 1, 128, 16, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("nq,lens", LENS)
@pytest.mark.parametrize("dtype,hq,hkv,d,block,by_token", LAYOUTS)
def test_attention_of_new_tokens(nq, lens, dtype, hq, hkv, d, block, by_token):
    cache, pools, table, status, q = _case(nq, lens, hq, hkv, d, block, dtype, 40 + len(nq), by_token, mb=-(-max(lens) // block) + 3)
    for causal in (True, False):
        out, lse = cache.attn(q, _i32(lens), _cu(nq), max_q=max(nq), max_len=max(max(lens), 1), causal=causal, return_lse=True)
        _check_attn(out, lse, q, pools, table, lens, nq, causal, dtype)
        out, lse = cache.attn(q, _i32(lens), _cu(nq), causal=causal, return_lse=True)  # bounds from the shapes
        _check_attn(out, lse, q, pools, table, lens, nq, causal, dtype)
        if all(m == 1 for m in nq):
            one, lse1 = cache.attn(q, _i32(lens), max_len=max(lens), causal=causal, return_lse=True)
            _check_attn(one, lse1, q, pools, table, lens, nq, causal, dtype)
    assert int(status) == 0
