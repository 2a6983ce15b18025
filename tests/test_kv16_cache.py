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
    (dict(out=4096, out_stride=(512, 64)), 1, "its strides"),
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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,hq,hkv,d,block", [
    (torch.bfloat16, 28, 4, 128, 64), (torch.float16, 16, 1, 128, 32), (torch.bfloat16, 8, 8, 64, 16), (torch.float16, 40, 1, 64, 128), (torch.bfloat16, 37, 1, 128, 16),
    (torch.float16, 64, 2, 64, 64), (torch.bfloat16, 6, 3, 128, 128),
])
@pytest.mark.parametrize("nq,lens", [([1, 1], [900, 77]), ([2, 2], [1500, 130]), ([5, 3], [700, 4]), ([16, 17], [2000, 300]), ([150], [1111])])
def test_head_layouts(dtype, hq, hkv, d, block, nq, lens):
    cache, pools, table, status, q = _case(nq, lens, hq, hkv, d, block, dtype, 50)
    out, lse = cache.attn(q, _i32(lens), _cu(nq), max_q=max(nq), max_len=max(lens), return_lse=True)
    _check_attn(out, lse, q, pools, table, lens, nq, True, dtype)
    assert int(status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("gain", [0.02, 8.0])
@pytest.mark.parametrize("nq,lens", [([1, 3], [700, 1300]), ([200], [900])])
def test_flat_and_sharp_distributions(gain, nq, lens):
    cache, pools, table, _, q = _case(nq, lens, 4, 2, 128, 32, torch.bfloat16, 51, gain=gain)
    out, lse = cache.attn(q, _i32(lens), _cu(nq), return_lse=True)
    _check_attn(out, lse, q, pools, table, lens, nq, True, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("nq", [1, 40, 500])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_logits_that_grow_along_the_keys_move_the_reference(nq, sign):
    n, hkv, d, block, dtype = 3000, 1, 128, 16, torch.float16
    cache, pools, table, _, q = _case([nq], [n], 2, hkv, d, block, dtype, 52)
    slope = sign * torch.linspace(-3, 3, n, device="cuda")
    for t in range(0, n, block):
        page = int(table[0, t // block])
        m = min(block, n - t)
        pools[0][page, 0, :m] = (pools[0][page, 0, :m].float() * 0.1 + slope[t:t + m, None]).to(dtype)
    q = (q.float() * 0.1 + 1.0).to(dtype)
    out, lse = cache.attn(q, _i32([n]), _cu([nq]), max_q=nq, return_lse=True)
    _check_attn(out, lse, q, pools, table, [n], [nq], True, dtype)


@pytest.mark.gpu
def test_an_own_softmax_scale():
    for nq in (1, 60):
        cache, pools, table, _, q = _case([nq], [500], 4, 2, 64, 16, torch.float16, 53)
        out, lse = cache.attn(q, _i32([500]), _cu([nq]), softmax_scale=0.37, return_lse=True)
        _check_attn(out, lse, q, pools, table, [500], [nq], True, torch.float16, scale=0.37)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,lens", [([1], [9000]), ([1, 1, 1], [40000, 130, 5000]), ([7], [30000]), ([1, 40, 3], [20000, 6001, 90]), ([300, 1], [9000, 30000])])
@pytest.mark.parametrize("dtype,hq,hkv,d,block", [(torch.bfloat16, 4, 2, 128, 64), (torch.float16, 7, 1, 64, 16)])
def test_long_contexts_are_shared_by_many_thread_blocks(nq, lens, dtype, hq, hkv, d, block):
    cache, pools, table, _, q = _case(nq, lens, hq, hkv, d, block, dtype, 54)
    args = dict(cu_q=_cu(nq), max_q=max(nq), max_len=max(lens), return_lse=True)
    for causal in (True, False):
        out, lse = cache.attn(q, _i32(lens), causal=causal, **args)
        _check_attn(out, lse, q, pools, table, lens, nq, causal, dtype)
    again, lse2 = cache.attn(q, _i32(lens), causal=False, **args)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def _fill_pages(pools, table, s, k, v, block):
    """Puts keys and values [n, H, d] of sequence s into its pages."""
    for w, x in enumerate((k, v)):
        for t in range(0, x.shape[0], block):
            m = min(block, x.shape[0] - t)
            pools[w][int(table[s, t // block]), :, :m] = x[t:t + m].transpose(0, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nk,hq,hkv,d,dtype,block", [
    (1, 16000, 4, 2, 128, torch.bfloat16, 64), (2, 70000, 4, 2, 128, torch.bfloat16, 64), (1, 70000, 7, 1, 64, torch.float16, 16), (40, 24001, 4, 1, 128, torch.float16, 32),
    (300, 9000, 2, 1, 64, torch.bfloat16, 128),
])
def test_shared_keys_lose_and_exchange_no_part(nq, nk, hq, hkv, d, dtype, block):
    from test_prompt_attn import _check_rms, _part_keys

    g = torch.Generator().manual_seed(71)
    q, v = torch.randn((nq, hq, d), generator=g).to(dtype).cuda(), torch.randn((nk, hkv, d), generator=g).to(dtype).cuda()
    k = _part_keys(nk, hkv, d, 16, dtype, g).cuda()
    cache, pools, table, _ = _cache([nk], hkv, d, block, dtype, 72)
    _fill_pages(pools, table, 0, k, v, block)
    _check_rms(cache.attn(q, _i32([nk]), _cu([nq]), max_q=nq, max_len=nk), q, k, v, True, dtype, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("nq,lens", [([1, 1, 1, 1], [1000, 600, 40, 2500]), ([9, 30, 2, 1], [1000, 600, 40, 2500]), ([300], [1500])])
def test_blocks_that_are_not_there_are_not_attended_to(nq, lens, block):
    hq, hkv, d, dtype = 4, 2, 128, torch.bfloat16
    cache, pools, table, status, q = _case(nq, lens, hq, hkv, d, block, dtype, 55)
    rng = np.random.default_rng(block)
    for holes in (0.2, 0.9, 1.0):
        gaps = np.where(rng.random(table.shape) < holes, -1, table).astype(np.int32)
        gaps[0, :1] = table[0, :1]  # (a sequence that keeps its first block alone)
        view = binding.Kv16Cache(pools[0], pools[1], torch.tensor(gaps, device="cuda"), status)
        for max_len in (max(lens), 100000):
            if max_len > gaps.shape[1] * block:
                max_len = gaps.shape[1] * block
            out, lse = view.attn(q, _i32(lens), _cu(nq), max_q=max(nq), max_len=max_len, return_lse=True)
            _check_attn(out, lse, q, pools, gaps, lens, nq, True, dtype)
    assert int(status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("nq,n", [(1, 500), (1, 50000), (200, 2000)])
@pytest.mark.parametrize("wrong", [-2, -2 ** 31, 2 ** 31 - 1, None])
def test_impossible_pages_are_absent_and_said(nq, n, wrong):
    hq, hkv, d, block, dtype = 4, 2, 64, 32, torch.float16
    cache, pools, table, status, q = _case([nq], [n], hq, hkv, d, block, dtype, 56)
    table = table.copy()
    table[0, 3] = table[0, -1] = pools[0].shape[0] if wrong is None else wrong
    view = binding.Kv16Cache(pools[0], pools[1], torch.tensor(table, device="cuda"), status)
    out, lse = view.attn(q, _i32([n]), _cu([nq]), max_q=nq, return_lse=True)
    _check_attn(out, lse, q, pools, table, [n], [nq], True, dtype)
    assert int(status) == 10


@pytest.mark.gpu
@pytest.mark.parametrize("nq,lens", [([4, 1], [70, 9]), ([70, 9], [70, 9]), ([3, 1], [41000, 900])])
def test_what_lies_outside_the_sequences_is_neither_used_nor_written(nq, lens):
    hq, hkv, d, block, dtype = 4, 2, 128, 32, torch.bfloat16
    cache, pools, table, status, _ = _case(nq, lens, hq, hkv, d, block, dtype, 57)
    q = _rows(5 + sum(nq) + 50, hq, d, dtype, 58)
    q[:5], q[5 + sum(nq):] = float("nan"), float("inf")
    out, before = torch.full_like(q, 3.0), [x.clone() for x in pools]
    got, lse = cache.attn(q, _i32(lens), _cu(nq, 5), max_q=max(nq), max_len=max(lens), out=out, return_lse=True)
    assert got is out
    _check_attn(out, lse, q, pools, table, lens, nq, True, dtype, 5)
    a, b = 5, 5 + sum(nq)
    assert (out[:a] == 3).all() and (out[b:] == 3).all() and int(status) == 0
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(pools, before))
    one = cache.attn(q[:7], _i32(lens), out=out[:7])  # without bounds: one token each, rows of nobody behind
    assert (one[2:5] == 3).all()


@pytest.mark.gpu
def test_a_sequence_has_the_same_bits_whatever_values_are_next_to_it():
    hq, hkv, d, block, dtype = 6, 2, 128, 16, torch.bfloat16
    for nq, lens in (([1, 1, 1], [900, 16, 4000]), ([37, 3, 150], [900, 16, 4000]), ([2, 1, 1], [900, 16, 60000])):
        cache, pools, table, _, q = _case(nq, lens, hq, hkv, d, block, dtype, 59, gain=4.0)
        args = dict(cu_q=_cu(nq), max_q=max(nq), max_len=max(lens), return_lse=True)
        alone = cache.attn(q, _i32(lens), **args)
        for fill in (1e4, float("nan"), float("inf")):
            q2 = q.clone()
            q2[nq[0]:nq[0] + nq[1]] = fill
            for x in pools:
                x[int(table[1, 0])] = fill
            out, lse = cache.attn(q2, _i32(lens), **args)
            for a, b in ((0, nq[0]), (nq[0] + nq[1], sum(nq))):
                assert torch.equal(out[a:b], alone[0][a:b]) and torch.equal(lse[:, a:b], alone[1][:, a:b])


@pytest.mark.gpu
@pytest.mark.parametrize("max_q,max_len,lens,cu,rows,code", [
    (4, 600, [600, 90], [0, 4, 6], 6, 0), (3, 600, [600, 90], [0, 4, 6], 6, 11), (4, 599, [600, 90], [0, 4, 6], 6, 11), (4, 600, [-1, 90], [0, 4, 6], 6, 11),
    (4, 600, [600, 90], [0, 4, 3], 6, 11), (4, 600, [600, 90], [0, 4, 8], 6, 11), (4, 600, [600, 90], [-2, 4, 6], 6, 11), (4, 10 ** 6, [10 ** 6, 90], [0, 4, 6], 6, 11),
    (2 ** 31 - 1025, 2 ** 31 - 1, [600, 90], [0, 4, 6], 6, 0),
])
def test_lengths_and_bounds_that_are_cut_set_the_status(max_q, max_len, lens, cu, rows, code):
    hq, hkv, d, block, dtype = 2, 1, 64, 16, torch.float16
    for more in (1, 40):  # few rows, and tiles of them
        true = [608, 96]
        cache, pools, table, status = _cache(true, hkv, d, block, dtype, 60)
        n_rows = rows * more
        q = _rows(n_rows, hq, d, dtype, 61)
        bounds = [c * more for c in cu]
        mq = max_q * more if max_q < 1000 else max_q
        out, lse = cache.attn(q, _i32(lens), _i32(bounds), max_q=mq, max_len=max_len, out=torch.full_like(q, 3.0), return_lse=True)
        assert int(status) == code, int(status)
        cap = min(table.shape[1] * block, max_len)
        pages = oracle.Pages([_np(x) for x in pools], table)
        for s in range(2):
            a, b = max(0, min(bounds[s], n_rows)), min(bounds[s + 1], n_rows)
            if b <= a or (code and s == 1 and cu[1] > cu[2]):
                continue
            m, n = min(b - a, mq), max(0, min(lens[s], cap))
            k, v, places = pages.rows(s, n)
            _check_seq(out[a:a + m], lse[:, a:a + m], q[a:a + m], k, v, n, places, True, dtype, (more, s))


@pytest.mark.gpu
@pytest.mark.parametrize("n_seqs", [33, 700])
@pytest.mark.parametrize("most", [1, 3, 90])
def test_many_sequences(n_seqs, most):
    hq, hkv, d, block, dtype = 4, 2, 64, 16, torch.bfloat16
    rng = np.random.default_rng(n_seqs + most)
    nq = rng.integers(0, most + 1, n_seqs)
    lens = nq + rng.integers(0, 200, n_seqs)
    lens[5], nq[7], lens[9] = 3000, most, 0
    cache, pools, table, status, q = _case(list(nq), list(lens), hq, hkv, d, block, dtype, 62)
    out, lse = cache.attn(q, _i32(lens), _cu(nq), max_q=most, max_len=int(max(lens)), return_lse=True)
    _check_attn(out, lse, q, pools, table, [int(x) for x in lens], [int(x) for x in nq], True, dtype)
    assert int(status) == 0


@pytest.mark.gpu
def test_as_many_sequences_as_a_call_takes():
    n, hq, hkv, d, block, dtype = 65535, 2, 1, 64, 16, torch.float16
    g = torch.Generator().manual_seed(63)
    pools = [torch.randn((50, hkv, block, d), generator=g).to(dtype).cuda() for _ in range(2)]
    table = torch.randint(0, 50, (n, 2), generator=g, dtype=torch.int32)
    lens = torch.randint(0, 33, (n,), generator=g, dtype=torch.int32)
    q = _rows(n, hq, d, dtype, 64)
    cache = binding.Kv16Cache(pools[0], pools[1], table.cuda())
    out, lse = cache.attn(q, lens.cuda(), return_lse=True)
    pages = oracle.Pages([_np(x) for x in pools], table.numpy())
    for s in (0, 1, 31, 32, 40000, 65533, 65534):
        k, v, places = pages.rows(s, int(lens[s]))
        _check_seq(out[s:s + 1], lse[:, s:s + 1], q[s:s + 1], k, v, int(lens[s]), places, True, dtype, s)
    empty = (lens == 0).cuda()
    assert not out[empty].any() and torch.isneginf(lse[:, empty]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("nq", [1, 50])
def test_pages_past_2_to_the_31_elements(nq):
    hq, hkv, d, block, dtype = 16, 8, 128, 128, torch.float16
    n_pages = (1 << 31) // (hkv * d * block) + 40
    pools = [torch.zeros((n_pages, hkv, block, d), dtype=dtype, device="cuda") for _ in range(2)]
    table = np.array([[n_pages - 1, 0, n_pages - 30, n_pages - 2]], np.int32)
    for x in pools:
        for p in table[0]:
            x[int(p)] = _rows(hkv * block, 1, d, dtype, int(p) % 97)[:, 0].view(hkv, block, d)
    cache = binding.Kv16Cache(pools[0], pools[1], torch.tensor(table, device="cuda"))
    q = _rows(nq, hq, d, dtype, 65)
    out, lse = cache.attn(q, _i32([500]), _cu([nq]), max_q=nq, return_lse=True)
    small = [torch.stack([x[int(p)] for p in table[0]]) for x in pools]
    _check_attn(out, lse, q, small, np.arange(4)[None], [500], [nq], True, dtype)


def _strided(how, n_pages, hkv, block, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    shapes = {"pairs": (n_pages, 2, hkv, block, d), "by token": (n_pages, block, hkv, d), "padded heads": (n_pages, block, hkv, d + 8), "padded rows": (n_pages, hkv, block, d + 8),
              "heads first": (hkv, n_pages, block, d)}
    pools = [torch.randn(shapes[how], generator=g).to(dtype).cuda() for _ in range(1 if how == "pairs" else 2)]
    if how == "pairs":
        return [pools[0][:, 0], pools[0][:, 1]]
    if how == "heads first":
        return [x.transpose(0, 1) for x in pools]
    if how == "padded rows":
        return [x[..., :d] for x in pools]
    return [x[..., :d].transpose(1, 2) for x in pools]


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["pairs", "by token", "padded heads", "padded rows", "heads first"])
@pytest.mark.parametrize("nq", [2, 90])
@pytest.mark.parametrize("d,block,dtype", [(128, 16, torch.bfloat16), (64, 128, torch.float16)])
def test_strides_of_the_pages(how, nq, d, block, dtype):
    hq, hkv, n = 6, 3, 700
    n_pages = -(-n // block) + 3
    pools = _strided(how, n_pages, hkv, block, d, dtype, 66)
    before = [x.clone() for x in pools]
    table = np.random.default_rng(67).permutation(n_pages)[None, :-(-n // block)].astype(np.int32)
    cache = binding.Kv16Cache(pools[0], pools[1], torch.tensor(table, device="cuda"))
    k, v = _rows(nq, hkv, d, dtype, 68), _rows(nq, hkv, d, dtype, 69)
    cache.append(k, v, _i32([n - nq]), cu_new=_cu([nq]))
    _check_append(cache, pools, table, before, k, v, [n - nq], [nq], [0], _np(k), np.zeros(k.shape))
    wide = _rows(nq, hq + 2, d + 8, dtype, 70)
    q, out = wide[:, 1:hq + 1, 8:], torch.empty((hq, nq, d), dtype=dtype, device="cuda").transpose(0, 1)
    got, lse = cache.attn(q, _i32([n]), _cu([nq]), out=out, return_lse=True)
    assert got is out
    _check_attn(out, lse, q, pools, table, [n], [nq], True, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,lens", [([2, 1], [700, 90]), ([1, 3], [60000, 90]), ([333, 90], [333, 900]), ([3000], [3100])])
def test_the_output_may_take_the_place_of_the_queries(nq, lens):
    cache, _, _, _, q = _case(nq, lens, 8, 2, 128, 64, torch.bfloat16, 73)
    args = dict(cu_q=_cu(nq), max_q=max(nq), max_len=max(lens))
    want = cache.attn(q, _i32(lens), **args)
    got = cache.attn(q, _i32(lens), out=q, **args)
    assert got is q and torch.equal(q, want)


@pytest.mark.gpu
def test_many_work_items_are_handed_out_whole():
    # more than six items for each SM: 64 heads of their own KV head; sequences with one tile of rows among them
    nq, lens, hq, d, dtype = [4100, 1, 3, 128], [4500, 3000, 100, 700], 64, 64, torch.float16
    cache, pools, table, _, q = _case(nq, lens, hq, hq, d, 128, dtype, 74)
    out, lse = cache.attn(q, _i32(lens), _cu(nq), return_lse=True)
    at = 0
    for s, (m, n) in enumerate(zip(nq, lens)):
        rows = [torch.cat([x[int(p)] for p in table[s, :-(-n // 128)]], dim=1)[:, :n].transpose(0, 1) for x in pools]
        for h in (0, 17, 63):
            _check_seq(out[at:at + m, h:h + 1], lse[h:h + 1, at:at + m], q[at:at + m, h:h + 1], _np(rows[0][:, h:h + 1]), _np(rows[1][:, h:h + 1]), n, None, True, dtype, (s, h))
        at += m


# ---- the operators together ------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,hq,hkv,d,block,n_axes", [(torch.bfloat16, 8, 2, 128, 16, 1), (torch.float16, 6, 3, 64, 64, 3)])
def test_prompts_in_pieces_then_drafts_then_tokens(dtype, hq, hkv, d, block, n_axes):
    """Two sequences as a server takes them, against the attention of whole prompts over keys rotated by themselves."""
    rotation, _ = _spec(d // 2, n_axes)
    total = [410, 300]
    qkv = [[_rows(n, h, d, dtype, 80 + s) for h in (hq, hkv, hkv)] for s, n in enumerate(total)]
    pos = [_i32(np.random.default_rng(s).integers(0, 9999, (n_axes, n))) if n_axes > 1 else _i32(np.arange(n))[None] for s, n in enumerate(total)]
    whole = []
    for (q, k, v), p, n in zip(qkv, pos, total):
        rq, rk = binding.qevict_rope(q, p, rotation, k=k)
        whole.append((binding.qevict_prompt_attn(rq, rk, v, _cu([n]), return_lse=True), rq, rk, v))
    cache = binding.Kv16Cache.allocate(80, 2, 32, hkv, d, block, dtype)
    cache.block_table.copy_(torch.randperm(80, generator=torch.Generator().manual_seed(1))[:64].view(2, 32).to(torch.int32))
    at = [0, 0]
    out = [torch.zeros_like(x[0]) for x in qkv]
    for step in ([200, 90], [150, 200], [5, 3], [1, 0], [0, 1], [4, 6], [50, 0]):
        take = [slice(a, a + m) for a, m in zip(at, step)]
        q, k, v = (torch.cat([x[i][t] for x, t in zip(qkv, take)]) for i in range(3))
        start, cu = _i32(at), _cu(step)
        p = torch.cat([x[:, t] for x, t in zip(pos, take)], dim=1) if n_axes > 1 else None
        rq = cache.append(k, v, start, cu_new=cu, rotation=rotation, positions=p, q=q)
        got = cache.attn(rq, start + cu.diff(), cu_q=cu, max_q=max(step))
        for s, part in enumerate(got.split(step)):
            out[s][take[s]] = part
        at = [a + m for a, m in zip(at, step)]
    assert at == total and int(cache.status) == 0
    for s, ((_, lse), rq, rk, v) in enumerate(whole):
        _check_seq(out[s], lse, rq, _np(rk), _np(v), total[s], None, True, dtype, s)
    # a draft that is not accepted: the sequence is cut back and goes on
    again = cache.attn(whole[0][1][190:200].contiguous(), _i32([200, 0]), cu_q=_cu([10, 0]))
    want = prompt.attention(_np(whole[0][1][190:200]), _np(whole[0][2][:200]), _np(whole[0][3][:200]), True)
    tol = prompt.out_tolerance(want[0], want[2], float(whole[0][3].abs().max()), 200, d, want[3], HALF_STEP[dtype], HALF_STEP[dtype])
    assert (np.abs(_np(again) - want[0]) <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("nq,room", [(1, 600), (1, 40000), (30, 600)])
def test_captured_with_the_lengths_advanced_inside(nq, room):
    hq, hkv, d, block, dtype, n = 4, 2, 128, 64, torch.bfloat16, 2
    rotation, _ = _spec(64)
    cache, pools, table, status = _cache([room] * n, hkv, d, block, dtype, 90)
    q, k, v = (_rows(n * nq, h, d, dtype, 91 + i) for i, h in enumerate((hq, hkv, hkv)))
    first = [100, room - 10 * nq]
    lens, cu = _i32(first), _cu([nq] * n)
    graphs, outs = [], []
    for _ in range(2):  # two graphs of the same step
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            rq = cache.append(k, v, lens, cu_new=cu, rotation=rotation, q=q)
            lens += nq
            outs.append(cache.attn(rq, lens, cu_q=cu, max_q=nq, max_len=room, return_lse=True))
        graphs.append((graph, rq))
    for step in range(4):
        k.copy_(_rows(n * nq, hkv, d, dtype, 95 + step))
        graph, rq = graphs[step % 2]
        graph.replay()
        out, lse = outs[step % 2]
        _check_attn(out, lse, rq, pools, table, [f + (step + 1) * nq for f in first], [nq] * n, True, dtype)
    assert int(status) == 0


@pytest.mark.gpu
def test_two_calls_at_once_and_on_another_stream():
    cases = [_case(nq, lens, 8, 2, 128, 32, torch.bfloat16, 100 + i) for i, (nq, lens) in enumerate((([1, 2], [30000, 700]), ([500], [2000]), ([1], [300])))]
    calls = [(c[0], c[4], _i32(lens), _cu(nq)) for c, (nq, lens) in zip(cases, (([1, 2], [30000, 700]), ([500], [2000]), ([1], [300])))]
    want = [c.attn(q, lens, cu) for c, q, lens, cu in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, (c, q, lens, cu) in zip(streams, calls):
            got.append(c.attn(q, lens, cu, stream=s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_the_first_call_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import torch
from paper_2608_05326_b200 import binding
cache = binding.Kv16Cache.allocate(70, 1, 64, 2, 64, 128, torch.float16)
cache.block_table.copy_(torch.arange(64, dtype=torch.int32)[None])
g = torch.Generator().manual_seed(1)
k, v = (torch.randn((1300, 2, 64), generator=g).half().cuda() for _ in range(2))
q = torch.randn((1300, 4, 64), generator=g).half().cuda()
rotation = binding.Rotation.standard(64)
start, lens, cu = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0], [1300], [0, 1300]))
few = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    rq = cache.append(k, v, start, cu_new=cu, rotation=rotation, q=q)
    out = cache.attn(rq, lens, cu_q=cu)
    last = cache.attn(rq[-1:], lens, cu_q=few, max_q=1, max_len=1300)
graph.replay()
again = cache.attn(rq, lens, cu_q=cu)
one = cache.attn(rq[-1:], lens, cu_q=few, max_q=1, max_len=1300)
assert torch.equal(out, again) and torch.equal(last, one) and out.abs().sum() > 0
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=root, timeout=600)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout[-1000:] + r.stderr[-3000:]


@pytest.mark.gpu
def test_nothing_to_attend_to_and_nothing_to_do():
    cache, pools, table, status = _cache([64, 64], 2, 64, 16, torch.float16, 110)
    q = _rows(40, 4, 64, torch.float16, 111)
    for cu, mq in (([0, 1, 2], 1), ([0, 20, 40], 20)):
        rows = cu[-1]
        out, lse = cache.attn(q[:rows], _i32([0, 0]), _i32(cu), max_q=mq, return_lse=True)
        assert not out.any() and torch.isneginf(lse).all()
    for args in (dict(cu_q=_i32([0, 0, 0])), dict(max_q=0, cu_q=_i32([0, 20, 40]))):
        out = cache.attn(q, _i32([64, 64]), out=torch.full_like(q, 3.0), **args)
        assert (out == 3).all()
    out = cache.attn(q[:2], _i32([64, 64]), max_len=0)
    assert not out.any() and int(status) == 11
    assert cache.attn(q[:0], _i32([64, 64]), cu_q=_i32([0, 0, 0])).shape == (0, 4, 64)


@pytest.mark.gpu
def test_attention_of_the_binding_refuses_what_the_library_cannot_see():
    cache = binding.Kv16Cache.allocate(4, 2, 2, 2, 64, 16, torch.float16)
    q, lens, cu = _rows(2, 4, 64, torch.float16, 2), _i32([0, 0]), _i32([0, 1, 2])
    for bad in (lambda: cache.attn(q.float(), lens), lambda: cache.attn(q[0], lens), lambda: cache.attn(q[..., :32], lens), lambda: cache.attn(q, lens[:1]),
                lambda: cache.attn(q, lens.long()), lambda: cache.attn(q, lens, cu_q=lens), lambda: cache.attn(q, lens, out=q[:1]), lambda: cache.attn(q, lens, out=q.bfloat16()),
                lambda: cache.attn(q, lens, max_q=2 ** 40), lambda: cache.attn(q, lens, max_len="a"), lambda: cache.attn(q, lens, max_q=2), lambda: cache.attn(q[:1], lens),
                lambda: cache.attn(q, lens, cu_q=cu, softmax_scale=-1.0), lambda: cache.attn(q[:, :3], lens), lambda: cache.attn(q.transpose(1, 2), lens)):
        with pytest.raises(binding.QEvictError):
            bad()


# ---- bounds that fall and rise ---------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("n_seqs,total,n,causal", [(200, 4096, 40000, False), (64, 4096, 140000, True), (9, 700, 5000, True)])
def test_bounds_that_give_many_sequences_the_same_rows(n_seqs, total, n, causal):
    # 0, total, 0, total, ...: every second sequence falls and is empty, every other one has all rows.  Their work together passes 2^32 of
    # the units in which it is shared out, although the rows of the call alone would not (the last case: both fit).  All have the
    # same pages, so whichever of them a row's result is from, it is the same but for its sums' order.
    hq, hkv, d, block, dtype = 32, 8, 64, 128, torch.bfloat16
    blocks = -(-n // block)
    pools = [torch.randn((blocks, hkv, block, d), generator=torch.Generator().manual_seed(120 + w)).to(dtype).cuda() for w in range(2)]
    table = torch.randperm(blocks, generator=torch.Generator().manual_seed(122)).to(torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = binding.Kv16Cache(pools[0], pools[1], table[None].repeat(n_seqs, 1).cuda(), status)
    q = _rows(total + 1, hq, d, dtype, 123)
    cu = [total * (i % 2) for i in range(n_seqs + 1)]
    out, lse = cache.attn(q, _i32([n] * n_seqs), _i32(cu), max_q=total, max_len=n, causal=causal, out=torch.full_like(q, 3.0), return_lse=True)
    assert int(status) == 11
    assert (out[total:] == 3).all()
    k, v = ((x[table.long().cuda()].transpose(0, 1).reshape(hkv, -1, d)[:, :n].transpose(0, 1)) for x in pools)
    for row in (0, 1, total // 3, total // 2 + 5, total - 1):
        for g in (0, 5):
            h, seen = slice(g * 4, g * 4 + 4), n - total + row + 1 if causal else n
            _check_seq(out[row:row + 1, h], lse[h, row:row + 1], q[row:row + 1, h], _np(k[:seen, g:g + 1]), _np(v[:seen, g:g + 1]), seen, None, False, dtype, (row, g))
    assert out.isfinite().all() and lse[:, :total].isfinite().all()


def test_more_work_items_than_a_search_can_add_up_are_refused():
    # 32 sequences may each have all rows of the call where bounds fall and rise: their items together have to stay below 2^31
    view = _view(n_kv_heads=32, k_stride=(32768, 1024, 64), v_stride=(32768, 1024, 64), max_blocks=4096)
    for total, status in ((1 << 27, 4), (1 << 30, 4), ((1 << 31) - 1025, 4)):
        args = _attn_args(view, n_q_heads=32, total_q=total, max_q=total, max_len=65536, cu_q=4096, q_stride=(2048, 64), out_stride=(2048, 64))
        _refused(binding.lib().qevict_kv16_attn(C.byref(args), None, 0, None), status, "2^24 work items")


# ---- one sharp key and a long flat tail ------------------------------------------------------------------------
def _tail_keys(n, sinks, hkv, d, dtype, seed):
    """Every query (ones) has the logit 1.5625 d scale at the sinks, whose values are 0, and next to none elsewhere, where the values are
    about 1: with d = 128 a probability of 2^-25.5 of a sink's, with d = 64 and the scale of 128 doubled the same."""
    g = torch.Generator().manual_seed(seed)
    k, v = torch.randn((n, hkv, d), generator=g) * 0.01, 1.0 + 0.1 * torch.randn((n, hkv, d), generator=g)
    k[sinks], v[sinks] = 1.5625, 0.0
    return k.to(dtype).cuda(), v.to(dtype).cuda()


def _check_tail(out, lse, k, v, scale, dtype):
    """out [rows, Hq, d], lse [Hq, rows]: every row is a query of ones over all keys.

    A probability enters the product in 16 bits: half a step off, and in fp16, where the reference stands 2^7 below the
    largest logit, off by at most half the smallest subnormal, 2^-25, of 2^7 times the largest probability: 2^-32 of it.  bf16 has
    no such floor."""
    hq, d, hkv, n = out.shape[1], out.shape[2], k.shape[1], k.shape[0]
    wo, wl, spread, reach = prompt.attention(np.ones((1, hq, d)), _np(k), _np(v), False, scale)
    u = HALF_STEP[dtype]
    rel, floor = prompt.logit_error(d, reach), 2.0 ** -32 if dtype is torch.float16 else 0.0
    top = 1.0 / float(np.exp(wl[0, 0] - 1.5625 * d * scale))  # a sink's probability, the largest
    tol = 1.01 * u * np.abs(wo) + 1.01 * (u + rel) * spread + 1.01 * n * floor * top * float(v.double().abs().max()) + SMALLEST[dtype] / 2
    err = (out.double() - torch.tensor(wo, device=out.device)).abs() / torch.tensor(tol, device=out.device)
    assert float(err.max()) <= 1.0, float(err.max())
    assert ((lse.double() - torch.tensor(wl, device=out.device)).abs() <= torch.tensor(prompt.lse_tolerance(wl, d, reach), device=out.device)).all()
    assert hq % hkv == 0 and float((1.01 * u * np.abs(wo)).max()) < float(tol.max()) < 0.05 * float(np.abs(wo).max())  # the tail is seen


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,n_seqs,n,sinks", [
    (1, 3, 8000, [0, 16, 32, 48]),        # clusters: 16 keys for each of four warps in turn, the sinks before the tail
    (1, 222, 40000, [0, 16, 32, 48]),     # equal ranges
    (4, 111, 40000, [0, 16, 32, 48]),
    (30, 74, 40000, [20000, 39999]),      # pairs: the last tile first, one half of the keys each
    (100, 37, 40000, [39999]),            # tiles of rows
    (4096, 2, 40000, [39999]),
])
def test_a_long_flat_tail_under_a_sharp_key_is_not_lost(nq, n_seqs, n, sinks, d, dtype):
    hq, hkv, block = 8, 2, 128
    scale = 128 ** -0.5 * (2.0 if d == 64 else 1.0)
    k, v = _tail_keys(n, sinks, hkv, d, dtype, 130)
    blocks = -(-n // block)
    pools = [torch.zeros((blocks, hkv, block, d), dtype=dtype, device="cuda") for _ in range(2)]
    for x, y in zip(pools, (k, v)):
        x.copy_(torch.nn.functional.pad(y, (0, 0, 0, 0, 0, blocks * block - n)).view(blocks, block, hkv, d).transpose(1, 2))
    cache = binding.Kv16Cache(pools[0], pools[1], torch.arange(blocks, dtype=torch.int32, device="cuda")[None].repeat(n_seqs, 1))
    q = torch.ones((n_seqs * nq, hq, d), dtype=dtype, device="cuda")
    out, lse = cache.attn(q, _i32([n] * n_seqs), _cu([nq] * n_seqs), max_q=nq, causal=False, softmax_scale=scale, return_lse=True)
    _check_tail(out, lse, k, v, scale, dtype)
    if nq == 4096:  # the same kernel over keys side by side
        out, lse = binding.qevict_prompt_attn(q[:8192].contiguous(), k, v, _i32([0, 8192]), _i32([0, n]), causal=False, softmax_scale=scale, return_lse=True)
        _check_tail(out, lse, k, v, scale, dtype)
