"""Attention over whole prompts against a float64 evaluation, and what the call refuses."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import prompt as oracle
from paper_2608_05326_b200 import binding

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


# ---- refusals: checked before anything reaches a device --------------------------------------------------------
def _args(**over):
    a = binding.qevict_prompt_args()
    values = dict(struct_size=C.sizeof(a), device=0, dtype=1, layout=0, n_seqs=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_q=16,
                  max_k=16, causal=1, softmax_scale=0.0, total_q=32, total_k=32, q=4096, k=4096, v=4096, out=4096, q_bounds=4096, k_bounds=4096)
    values.update(over)
    for n, x in values.items():
        if n.endswith("_stride"):
            continue
        setattr(a, n, x)
    for n in ("q_stride", "k_stride", "v_stride", "out_stride"):
        heads = a.n_q_heads if n in ("q_stride", "out_stride") else a.n_kv_heads
        for i, x in enumerate(values.get(n, (0, 64, 64 * heads))):
            getattr(a, n)[i] = x
    return a


@pytest.mark.parametrize("over,status,word", [
    (dict(struct_size=8), 1, "struct_size"), (dict(device=-1), 1, "device"), (dict(dtype=7), 1, "dtype"), (dict(layout=2), 1, "layout"),
    (dict(causal=2), 1, "causal"), (dict(n_seqs=-1), 1, "sizes"), (dict(n_q_heads=7), 1, "multiple"), (dict(n_kv_heads=0), 1, "multiple"),
    (dict(softmax_scale=float("nan")), 1, "softmax_scale"), (dict(softmax_scale=-1.0), 1, "softmax_scale"), (dict(softmax_scale=1e-40), 1, "softmax_scale"), (dict(head_dim=96), 4, "head_dim"),
    (dict(q=None), 1, "NULL"), (dict(k=None), 1, "NULL"), (dict(out=None), 1, "NULL"), (dict(q_bounds=None), 1, "q_bounds"),
    (dict(q=4104), 1, "aligned"), (dict(lse=4098), 1, "aligned"), (dict(k_stride=(0, 60, 128)), 1, "strides"),
    (dict(q_stride=(0, 64, 0)), 1, "strides"), (dict(total_q=2 ** 31), 4, "tokens"),
])
def test_unusable_arguments_are_refused_with_a_reason(over, status, word):
    with pytest.raises(binding.QEvictError) as e:
        binding._check(binding.lib().qevict_prompt_attn(C.byref(_args(**over)), None, 0, None))
    assert e.value.status == status and word in str(e.value)


@pytest.mark.parametrize("scale", [3e38, 2.5e38, float("inf"), float("nan"), -1e-3, 1e-31])
def test_scales_that_are_no_float_times_log2_e_are_refused(scale):
    lib, need = binding.lib(), C.c_uint64()
    for call in (lambda: lib.qevict_prompt_attn(C.byref(_args(softmax_scale=scale)), None, 0, None),
                 lambda: lib.qevict_prompt_attn_scratch_bytes(C.byref(_args(softmax_scale=scale)), C.byref(need))):
        assert call() == 1 and b"softmax_scale" in lib.qevict_last_error(None)
    assert lib.qevict_prompt_attn_scratch_bytes(C.byref(_args(softmax_scale=2e38)), C.byref(need)) == 0


def test_nothing_to_do_is_fine_without_a_device():
    lib = binding.lib()
    for over in (dict(n_seqs=0), dict(max_q=0), dict(total_q=0)):
        assert lib.qevict_prompt_attn(C.byref(_args(**over)), None, 0, None) == 0


def test_scratch_is_needed_only_for_few_queries_and_many_keys():
    lib, need = binding.lib(), C.c_uint64(1)
    binding._check(lib.qevict_prompt_attn_scratch_bytes(C.byref(_args()), C.byref(need)))
    assert need.value == 0
    few = _args(n_seqs=1, max_q=1, total_q=1, max_k=65536, total_k=65536)
    binding._check(lib.qevict_prompt_attn_scratch_bytes(C.byref(few), C.byref(need)))
    assert need.value > 0
    assert lib.qevict_prompt_attn(C.byref(few), None, 0, None) == 3  # QEVICT_ERR_NO_MEMORY
    assert b"scratch" in lib.qevict_last_error(None)
    assert lib.qevict_prompt_attn_scratch_bytes(C.byref(few), None) == 1


# ---- results ---------------------------------------------------------------------------------------------------
def _make(nq, nk, hq, hkv, d, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    q = (gain * torch.randn((sum(nq), hq, d), generator=g)).to(dtype)
    k = torch.randn((sum(nk), hkv, d), generator=g).to(dtype)
    v = torch.randn((sum(nk), hkv, d), generator=g).to(dtype)
    return q, k, v


def _cu(lens, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def _np(x):
    return x.double().cpu().numpy()


def _check_rows(out, lse, q, k, v, causal, dtype, what="", scale=None):
    """out [nq, Hq, d], lse [Hq, nq] of one sequence against the oracle."""
    ro, rl, spread, reach = oracle.attention(_np(q), _np(k), _np(v), causal, scale)
    d = q.shape[-1]
    vmax = float(v.double().abs().max()) if v.numel() else 0.0
    tol = oracle.out_tolerance(ro, spread, vmax, k.shape[0], d, reach, HALF_STEP[dtype], HALF_STEP[dtype])
    err = np.abs(_np(out) - ro)
    assert (err <= tol).all(), (what, float((err / tol).max()), float(err.max()))
    got = _np(lse)
    assert (np.isneginf(got) == np.isneginf(rl)).all(), what
    ok = np.isfinite(rl)
    assert np.isfinite(got[ok]).all() and (np.abs(got[ok] - rl[ok]) <= oracle.lse_tolerance(rl[ok], d, reach)).all(), what


def _check_packed(out, lse, q, k, v, nq, nk, causal, dtype, q_first=0, k_first=0, scale=None):
    a, b = q_first, k_first
    for i, (x, y) in enumerate(zip(nq, nk)):
        _check_rows(out[a:a + x], lse[:, a:a + x], q[a:a + x], k[b:b + y], v[b:b + y], causal, dtype, "sequence %d (%d, %d)" % (i, x, y), scale)
        a, b = a + x, b + y


LENS = [
    ([1], [1]), ([77], [77]), ([128], [128]), ([129], [129]), ([256], [256]), ([257], [257]), ([600], [600]),
    ([5, 0, 130, 1, 255], [5, 0, 130, 1, 255]), ([3, 200], [131, 456]), ([1, 64, 300], [700, 64, 301]),
    ([130, 4], [2, 3]), ([3, 2], [0, 2]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nk", LENS)
@pytest.mark.parametrize("dtype,hq,hkv,d", [(torch.bfloat16, 4, 2, 128), (torch.float16, 3, 1, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(nq, nk, dtype, hq, hkv, d, causal):
    q, k, v = (x.cuda() for x in _make(nq, nk, hq, hkv, d, dtype, 11 + len(nq)))
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), max(nq), max(nk), causal=causal, return_lse=True)
    _check_packed(out, lse, q, k, v, nq, nk, causal, dtype)
    again, lse2 = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), causal=causal, return_lse=True)  # bounds from the shapes
    _check_packed(again, lse2, q, k, v, nq, nk, causal, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,hq,hkv,d", [(torch.bfloat16, 28, 4, 128), (torch.float16, 8, 8, 64), (torch.bfloat16, 16, 1, 128), (torch.float16, 32, 8, 128)])
def test_head_layouts_and_longer_prompts(dtype, hq, hkv, d):
    nq = [1111, 517]
    q, k, v = (x.cuda() for x in _make(nq, nq, hq, hkv, d, dtype, 3))
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), max_q=max(nq), max_k=max(nq), return_lse=True)
    _check_packed(out, lse, q, k, v, nq, nq, True, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("gain", [0.02, 8.0])
def test_flat_and_sharp_distributions(gain):
    nq = [700]
    q, k, v = (x.cuda() for x in _make(nq, nq, 2, 1, 128, torch.bfloat16, 5, gain))
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), return_lse=True)
    _check_packed(out, lse, q, k, v, nq, nq, True, torch.bfloat16)


@pytest.mark.gpu
def test_logits_that_grow_along_the_keys_move_the_reference():
    # every tile of 128 keys has larger logits than all the ones behind it, and the reverse
    n, d = 1000, 128
    for sign in (1.0, -1.0):
        q, k, v = _make([n], [n], 1, 1, d, torch.float16, 9)
        k = k * 0.1 + (sign * torch.linspace(-3, 3, n)[:, None, None]).to(torch.float16)
        q = (q * 0.1 + 1.0).to(torch.float16)
        q, k, v = q.cuda(), k.to(torch.float16).cuda(), v.cuda()
        for causal in (True, False):
            out, lse = binding.qevict_prompt_attn(q, k, v, _cu([n]), causal=causal, return_lse=True)
            _check_packed(out, lse, q, k, v, [n], [n], causal, torch.float16)


@pytest.mark.gpu
def test_an_own_softmax_scale():
    nq = [300]
    q, k, v = (x.cuda() for x in _make(nq, nq, 2, 1, 64, torch.float16, 8))
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), softmax_scale=0.37, return_lse=True)
    _check_packed(out, lse, q, k, v, nq, nq, True, torch.float16, scale=0.37)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nk", [([1], [9000]), ([1, 3], [5000, 131]), ([40], [6001]), ([2], [70000])])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(torch.bfloat16, 4, 2, 128), (torch.float16, 7, 1, 64)])
def test_few_queries_behind_a_long_prefix_split_the_keys(nq, nk, dtype, hq, hkv, d):
    q, k, v = (x.cuda() for x in _make(nq, nk, hq, hkv, d, dtype, 21))
    args = dict(max_q=max(nq), max_k=max(nk), return_lse=True)
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), **args)
    _check_packed(out, lse, q, k, v, nq, nk, True, dtype)
    again, lse2 = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), **args)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nk", [([70, 9], [70, 9]), ([3, 1], [4100, 900])])
def test_what_lies_outside_the_sequences_is_neither_used_nor_written(nq, nk):
    d, hq, hkv, dtype = 128, 4, 2, torch.bfloat16
    q, k, v = (x.cuda() for x in _make([5] + nq + [200], [7] + nk + [200], hq, hkv, d, dtype, 2))
    for x, lo, hi in ((q, 5, 5 + sum(nq)), (k, 7, 7 + sum(nk)), (v, 7, 7 + sum(nk))):
        x[:lo] = float("nan")
        x[hi:hi + 100] = float("nan")
        x[hi + 100:] = float("inf")
    out = torch.full_like(q, 3.0)
    lse = torch.full((hq, q.shape[0]), 7.0, device="cuda")
    binding.qevict_prompt_attn(q, k, v, _cu(nq, 5), _cu(nk, 7), max(nq), max(nk), out=out, lse=lse)
    _check_packed(out, lse, q, k, v, nq, nk, True, dtype, 5, 7)
    a, b = 5, 5 + sum(nq)
    assert (out[:a] == 3).all() and (out[b:] == 3).all() and (lse[:, :a] == 7).all() and (lse[:, b:] == 7).all()


@pytest.mark.gpu
def test_one_sequence_does_not_reach_into_the_next():
    nq = [100, 150]
    q, k, v = (x.cuda() for x in _make(nq, nq, 2, 1, 64, torch.float16, 4))
    k[100:], v[100:] = float("nan"), float("inf")
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), return_lse=True)
    _check_rows(out[:100], lse[:, :100], q[:100], k[:100], v[:100], True, torch.float16)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,dtype", [(7, 1, 64, torch.float16), (6, 2, 128, torch.bfloat16), (1, 1, 128, torch.float16)])
def test_a_sequence_has_the_same_bits_whatever_is_next_to_it(hq, hkv, d, dtype):
    # rows of a tile that belong to nobody, or to another sequence, must not decide when a row's reference moves
    nq, nk = [37, 3, 150], [900, 3, 150]
    q, k, v = (x.cuda() for x in _make(nq, nk, hq, hkv, d, dtype, 33, 4.0))
    args = dict(max_q=150, max_k=900, return_lse=True)
    alone = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), **args)
    for fill in (1e4, float("nan"), float("inf")):
        q2, k2, v2 = q.clone(), k.clone(), v.clone()
        q2[37:40], k2[900:903], v2[900:903] = fill, fill, fill
        binding.qevict_prompt_attn(torch.full_like(q, fill), k, v, _cu(nq), _cu(nk), **args)  # leaves other values on the SMs
        out, lse = binding.qevict_prompt_attn(q2, k2, v2, _cu(nq), _cu(nk), **args)
        for a, b in ((0, 37), (40, 190)):
            assert torch.equal(out[a:b], alone[0][a:b]) and torch.equal(lse[:, a:b], alone[1][:, a:b])


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float16)])
def test_padded_layout_with_lengths(d, dtype):
    n, hq, hkv, m = 4, 4, 2, 300
    g = torch.Generator().manual_seed(1)
    q = torch.randn((n, hq, m, d), generator=g).to(dtype).cuda()
    k, v = (torch.randn((n, hkv, m + 20, d), generator=g).to(dtype).cuda() for _ in range(2))
    lq, lk = [300, 1, 0, 129], [320, 5, 3, 129]
    for i in range(n):
        for x, c in ((q, lq), (k, lk), (v, lk)):
            x[i, :, c[i]:] = float("nan")
    out = torch.full_like(q, 3.0)
    lse = torch.full((n, hq, m), 7.0, device="cuda")
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lq, lk)]
    binding.qevict_prompt_attn(q, k, v, lens[0], lens[1], out=out, lse=lse)
    for i in range(n):
        a, b = lq[i], lk[i]
        _check_rows(out[i, :, :a].transpose(0, 1), lse[i, :, :a], q[i, :, :a].transpose(0, 1), k[i, :, :b].transpose(0, 1), v[i, :, :b].transpose(0, 1), True, dtype)
        assert (out[i, :, a:] == 3).all() and (lse[i, :, a:] == 7).all()
    # without lengths every row counts
    q, k, v = torch.nan_to_num(q), torch.nan_to_num(k), torch.nan_to_num(v)
    out, lse = binding.qevict_prompt_attn(q, k, v, return_lse=True)
    for i in range(n):
        _check_rows(out[i].transpose(0, 1), lse[i], q[i].transpose(0, 1), k[i].transpose(0, 1), v[i].transpose(0, 1), True, dtype)


@pytest.mark.gpu
def test_strided_inputs_and_output():
    n, hq, hkv, d, dtype = 333, 4, 2, 128, torch.bfloat16
    g = torch.Generator().manual_seed(6)
    qkv = torch.randn((n, hq + 2 * hkv, d + 8), generator=g).to(dtype).cuda()  # one projection's output, rows padded
    q, k, v = qkv[:, :hq, :d], qkv[:, hq:hq + hkv, 8:], qkv[:, hq + hkv:, :d]
    buf = torch.zeros((hq, n, d), dtype=dtype, device="cuda")
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu([n]), out=buf.transpose(0, 1), return_lse=True)
    _check_rows(buf.transpose(0, 1), lse, q, k, v, True, dtype)
    plain = binding.qevict_prompt_attn(q.contiguous(), k.contiguous(), v.contiguous(), _cu([n]))
    assert torch.equal(plain, out)


def _rms(x):
    return float(np.sqrt(np.mean(np.square(x))))


def _check_rms(out, q, k, v, causal, dtype, parts):
    """The output of a long sequence within what independent roundings leave; and that a sum without one of `parts` equal parts of
    the keys, or with the weights of two neighbouring parts exchanged, would not be."""
    q, k, v = _np(q), _np(k), _np(v)
    ro, lse, _, reach = oracle.attention(q, k, v, causal)
    u = HALF_STEP[dtype]
    tol = oracle.rms_tolerance(ro, *oracle.roundings(q, k, v, causal), q.shape[-1], reach, u, u, dtype == torch.float16)
    assert _rms(_np(out) - ro) <= tol, _rms(_np(out) - ro) / tol
    n = k.shape[0] // parts
    for i in (0, parts // 2, parts - 2):
        a, b = slice(i * n, (i + 1) * n), slice((i + 1) * n, (i + 2) * n)
        part = []  # what a merge joins: output and log of the denominator of a part by itself
        for x in (a, b):
            o, l, _, _ = oracle.attention(q, k[x], v[x], False)  # (every query sees these keys)
            part.append((o, np.exp(l - lse).T[..., None]))
        (oa, wa), (ob, wb) = part
        assert _rms(oa * wa) > 3 * tol and _rms(ob * wb) > 3 * tol, i
        assert _rms(oa * (wb - wa) + ob * (wa - wb)) > 3 * tol, i


def _part_keys(n, hkv, d, parts, dtype, g):
    # neighbouring parts of the keys weigh differently: logits of small and of large spread in turn
    k = torch.randn((n, hkv, d), generator=g)
    return (k * torch.where(torch.arange(n) * parts // n % 2 == 0, 0.3, 1.2)[:, None, None]).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nk,hq,hkv,d,dtype", [
    (2, 70000, 4, 2, 128, torch.bfloat16), (1, 70000, 7, 1, 64, torch.float16), (40, 24001, 4, 1, 128, torch.float16), (300, 9000, 2, 1, 64, torch.bfloat16),
])
def test_split_keys_lose_and_exchange_no_part(nq, nk, hq, hkv, d, dtype):
    g = torch.Generator().manual_seed(71)
    q, v = torch.randn((nq, hq, d), generator=g).to(dtype), torch.randn((nk, hkv, d), generator=g).to(dtype)
    k = _part_keys(nk, hkv, d, 64, dtype, g)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu([nq]), _cu([nk]), return_lse=True)
    _check_packed(out, lse, q, k, v, [nq], [nk], True, dtype)
    _check_rms(out, q, k, v, True, dtype, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,dtype,causal", [(4, 2, 128, torch.bfloat16, True), (7, 1, 64, torch.float16, True), (4, 1, 64, torch.bfloat16, False)])
def test_padded_layout_with_split_keys(hq, hkv, d, dtype, causal):
    n, mq, mk = 3, 5, 20000
    g = torch.Generator().manual_seed(73)
    q = torch.randn((n, hq, mq, d), generator=g).to(dtype).cuda()
    v = torch.randn((n, hkv, mk, d), generator=g).to(dtype).cuda()
    k = torch.stack([_part_keys(mk, hkv, d, 16, dtype, g).transpose(0, 1) for _ in range(n)]).cuda()
    lq, lk = [5, 1, 3], [20000, 130, 11111]
    for i in range(n):
        for x, c in ((q, lq), (k, lk), (v, lk)):
            x[i, :, c[i]:] = float("nan")
    need, args = C.c_uint64(), _args(layout=1, n_seqs=n, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_q=mq, max_k=mk)
    binding._check(binding.lib().qevict_prompt_attn_scratch_bytes(C.byref(args), C.byref(need)))
    assert need.value > 0  # the keys are split
    out, lse = torch.full_like(q, 3.0), torch.full((n, hq, mq), 7.0, device="cuda")
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lq, lk)]
    binding.qevict_prompt_attn(q, k, v, lens[0], lens[1], causal=causal, out=out, lse=lse)
    for i in range(n):
        a, b = lq[i], lk[i]
        row = [x[i, :, :c].transpose(0, 1) for x, c in ((out, a), (q, a), (k, b), (v, b))]
        _check_rows(row[0], lse[i, :, :a], *row[1:], causal, dtype)
        if b > 1000:
            _check_rms(*row, causal, dtype, 16)
        assert (out[i, :, a:] == 3).all() and (lse[i, :, a:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,dtype", [(4, 2, 128, torch.bfloat16), (3, 1, 64, torch.float16)])
def test_long_prompts_within_independent_roundings(hq, hkv, d, dtype):
    n = 3001
    q, k, v = (x.cuda() for x in _make([n], [n], hq, hkv, d, dtype, 77))
    for causal in (True, False):
        out = binding.qevict_prompt_attn(q, k, v, _cu([n]), causal=causal)
        ro, _, _, reach = oracle.attention(_np(q), _np(k), _np(v), causal)
        u = HALF_STEP[dtype]
        tol = oracle.rms_tolerance(ro, *oracle.roundings(_np(q), _np(k), _np(v), causal), d, reach, u, u, dtype == torch.float16)
        assert _rms(_np(out) - ro) <= tol


@pytest.mark.gpu
def test_many_sequences_and_wide_groups():
    rng = np.random.default_rng(3)
    nq = [int(x) for x in rng.integers(0, 20, 150)]
    nk = [int(x + rng.integers(0, 90)) for x in nq]
    q, k, v = (x.cuda() for x in _make(nq, nk, 6, 3, 64, torch.float16, 12))
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), max(nq), max(nk), return_lse=True)
    _check_packed(out, lse, q, k, v, nq, nk, True, torch.float16)
    for hq, hkv in ((40, 1), (96, 2), (37, 1)):
        q, k, v = (x.cuda() for x in _make([70, 9], [70, 30], hq, hkv, 64, torch.bfloat16, 13))
        out, lse = binding.qevict_prompt_attn(q, k, v, _cu([70, 9]), _cu([70, 30]), 70, 70, return_lse=True)
        _check_packed(out, lse, q, k, v, [70, 9], [70, 30], True, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
def test_hundreds_of_sequences(causal):
    # several work items for every SM, several groups of 32 sequences, empty sequences at either end
    rng = np.random.default_rng(8)
    nq = [0, 0] + [int(x) for x in rng.integers(0, 300, 210)] + [700] + [int(x) for x in rng.integers(0, 40, 120)] + [0] * 40
    nk = [int(max(0, x + rng.integers(-20, 200))) for x in nq]
    q, k, v = (x.cuda() for x in _make(nq, nk, 4, 2, 64, torch.bfloat16, 14))
    out, lse = torch.full_like(q, 3.0), torch.full((4, sum(nq)), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), max(nq), max(nk), causal=causal, out=out, lse=lse, status=status)
    _check_packed(out, lse, q, k, v, nq, nk, causal, torch.bfloat16)
    assert int(status) == 0


@pytest.mark.gpu
def test_nothing_to_attend_to_and_nothing_to_do():
    q, k, v = (x.cuda() for x in _make([5], [0], 2, 1, 64, torch.float16, 1))
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu([5]), _cu([0]), return_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    out, lse = binding.qevict_prompt_attn(q[:0], k, v, _cu([0]), _cu([0]), return_lse=True)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    assert binding.qevict_prompt_attn(q, k, v, _cu([])[:1], return_lse=False).shape == q.shape  # no sequence


@pytest.mark.gpu
def test_lengths_are_cut_to_the_bounds():
    nq = [200, 90]
    q, k, v = (x.cuda() for x in _make(nq, nq, 2, 1, 64, torch.float16, 19))
    out = torch.full_like(q, 3.0)
    lse = torch.full((2, 290), 7.0, device="cuda")
    binding.qevict_prompt_attn(q, k, v, _cu(nq), max_q=150, max_k=140, causal=False, out=out, lse=lse)
    _check_rows(out[:150], lse[:, :150], q[:150], k[:140], v[:140], False, torch.float16)
    _check_rows(out[200:], lse[:, 200:], q[200:], k[200:], v[200:], False, torch.float16)
    assert (out[150:200] == 3).all() and (lse[:, 150:200] == 7).all()


def test_packed_bounds_beyond_the_rows_plan_like_the_rows():
    lib, need = binding.lib(), [C.c_uint64() for _ in range(2)]
    for args, n in zip((dict(max_q=40, max_k=70000), dict(max_q=1 << 29, max_k=1 << 30)), need):
        binding._check(lib.qevict_prompt_attn_scratch_bytes(C.byref(_args(total_q=40, total_k=70000, **args)), C.byref(n)))
    assert need[0].value == need[1].value > 0


@pytest.mark.gpu
@pytest.mark.parametrize("max_q,max_k", [(131072, 131072), (1 << 29, None), ((1 << 29) + 1, 1 << 30)])
def test_packed_bounds_beyond_the_rows(max_q, max_k):
    # one row in eight of 2^29 x 64 heads is 2^32 thread blocks: what a 32-bit grid cannot hold
    nq, nk = [1, 3, 2], [5000, 131, 900]
    q, k, v = (x.cuda() for x in _make(nq, nk, 64, 8, 64, torch.bfloat16, 51))
    out, lse = torch.full_like(q, 3.0), torch.full((64, 6), 7.0, device="cuda")
    binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), max_q, max_k, out=out, lse=lse)
    _check_packed(out, lse, q, k, v, nq, nk, True, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("cu_q,cu_k,max_q,max_k", [
    ([0, 20, 60], [0, 30, 90], 40, 60),     # as they should be
    ([0, 20, 61], [0, 30, 90], 60, 90),     # queries past the rows
    ([0, 20, 60], [0, 30, 200], 40, 90),    # keys past the rows
    ([-3, 20, 60], [0, 30, 90], 40, 60), ([0, 20, 60], [-1, 30, 90], 40, 60), ([0, 20, 7], [0, 30, 90], 40, 60), ([0, 20, 60], [0, 30, 9], 40, 60),
    ([0, 20, 60], [0, 30, 90], 39, 60), ([0, 20, 60], [0, 30, 90], 40, 59),
])
def test_packed_bounds_that_are_cut_set_the_status(cu_q, cu_k, max_q, max_k):
    q, _, _ = _make([60], [60], 2, 1, 64, torch.float16, 61)
    _, k, v = _make([90], [90], 2, 1, 64, torch.float16, 62)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    dev = dict(dtype=torch.int32, device="cuda")
    out, lse, status = torch.full_like(q, 3.0), torch.full((2, 60), 7.0, device="cuda"), torch.zeros(1, **dev)
    binding.qevict_prompt_attn(q, k, v, torch.tensor(cu_q, **dev), torch.tensor(cu_k, **dev), max_q, max_k, causal=False, out=out, lse=lse, status=status)
    cut = lambda c, most, total: [(max(0, a), min(b, total, max(0, a) + most)) for a, b in zip(c, c[1:])]  # noqa: E731
    seqs = list(zip(cut(cu_q, max_q, 60), cut(cu_k, max_k, 90)))
    written = torch.zeros(60, dtype=torch.bool)
    for (a, b), (x, y) in seqs:
        if b > a:
            y = max(x, y)
            _check_rows(out[a:b], lse[:, a:b], q[a:b], k[x:y], v[x:y], False, torch.float16)
            written[a:b] = True
    assert (out.cpu()[~written] == 3).all() and (lse.cpu()[:, ~written] == 7).all()
    good = (cu_q, cu_k, max_q, max_k) == ([0, 20, 60], [0, 30, 90], 40, 60)
    assert int(status) == (0 if good else 11)


@pytest.mark.gpu
@pytest.mark.parametrize("lq,lk,code", [([5, 9], [9, 0], 0), ([5, 10], [9, 0], 11), ([-1, 9], [9, 9], 11), ([5, 9], [9, 12], 11), (None, None, 0)])
def test_padded_lengths_that_are_cut_set_the_status(lq, lk, code):
    g = torch.Generator().manual_seed(63)
    q, k, v = (torch.randn((2, h, 9, 64), generator=g).half().cuda() for h in (2, 1, 1))
    dev = dict(dtype=torch.int32, device="cuda")
    out, lse, status = torch.full_like(q, 3.0), torch.full((2, 2, 9), 7.0, device="cuda"), torch.zeros(1, **dev)
    lens = [None if x is None else torch.tensor(x, **dev) for x in (lq, lk)]
    binding.qevict_prompt_attn(q, k, v, lens[0], lens[1], out=out, lse=lse, status=status)
    for i in range(2):
        a, b = (9 if x is None else min(max(x[i], 0), 9) for x in (lq, lk))
        _check_rows(out[i, :, :a].transpose(0, 1), lse[i, :, :a], q[i, :, :a].transpose(0, 1), k[i, :, :b].transpose(0, 1), v[i, :, :b].transpose(0, 1), True, torch.float16)
        assert (out[i, :, a:] == 3).all() and (lse[i, :, a:] == 7).all()
    assert int(status) == code


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nk", [([333, 1, 90], [333, 1, 90]), ([3, 2], [9000, 700])])
def test_the_output_may_take_the_place_of_the_queries(nq, nk):
    q, k, v = (x.cuda() for x in _make(nq, nk, 6, 2, 128, torch.bfloat16, 81))
    want, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), return_lse=True)
    got, lse2 = binding.qevict_prompt_attn(q, k, v, _cu(nq), _cu(nk), out=q, return_lse=True)
    assert got is q and torch.equal(got, want) and torch.equal(lse, lse2)


@pytest.mark.gpu
def test_padded_batch_without_keys():
    q = torch.randn((2, 2, 5, 64), device="cuda").half()
    k = torch.empty((2, 1, 0, 64), device="cuda").half()
    out, lse = binding.qevict_prompt_attn(q, k, k, return_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.gpu
def test_as_many_sequences_as_a_call_takes():
    # 65535 sequences of 0 to 2 tokens, a longer one among them
    n = 65535
    nq = np.random.default_rng(5).integers(0, 3, n)
    nq[[0, 40000, n - 1]] = [1, 150, 2]
    q, k, v = (x.cuda() for x in _make([int(nq.sum())], [int(nq.sum())], 2, 1, 64, torch.float16, 83))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = binding.qevict_prompt_attn(q, k, v, _cu(nq), max_q=150, max_k=150, return_lse=True, status=status)
    assert int(status) == 0
    cu = np.concatenate([[0], np.cumsum(nq)])
    one = torch.from_numpy(cu[:-1][nq == 1]).cuda()  # a row that sees itself alone
    assert torch.equal(out[one], v[one].expand(-1, 2, -1))
    for s in (40000, n - 1, 39999, 40001, 123, 65000):
        a, b = cu[s], cu[s + 1]
        _check_rows(out[a:b], lse[:, a:b], q[a:b], k[a:b], v[a:b], True, torch.float16)
    two = torch.from_numpy(cu[:-1][nq == 2]).cuda()
    x = [q[two + 1].double() * k[two + i].double() for i in range(2)]
    reach = max(float(y.abs().sum(-1).max()) / 8 for y in x)
    rl = torch.logaddexp(*(y.sum(-1) / 8 for y in x)).cpu().numpy()
    assert (np.abs(_np(lse[:, two + 1].T) - rl) <= oracle.lse_tolerance(rl, 64, reach)).all()


@pytest.mark.gpu
def test_the_first_call_of_a_process_may_be_captured():
    code = """
import torch
from paper_2608_05326_b200 import binding
q, k = torch.randn((40, 2, 64), device="cuda").half(), torch.randn((40, 1, 64), device="cuda").half()
i32 = dict(dtype=torch.int32, device="cuda")
cu, out, lens = torch.tensor([0, 40], **i32), torch.zeros_like(q), torch.tensor([3], **i32)
c = binding.Kv8Cache.allocate(4, 1, 4, 1, 64, 16, torch.float16)
c.block_table.copy_(torch.arange(4).view(1, 4))
acc, q1 = torch.zeros((1, 4), device="cuda"), q[:1].contiguous()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    binding.qevict_prompt_attn(q, k, k, cu, max_q=40, max_k=40, out=out)
    c.append(k, k, torch.zeros_like(lens), cu)
    got = c.attn(q1, lens, scores=acc, scores_out=acc)[0]
    ev = binding.qevict_kv8_evict(c.block_table, torch.full_like(lens, 40), acc, 16, 4, 1)
g.replay()
torch.cuda.synchronize()
assert torch.equal(out, binding.qevict_prompt_attn(q, k, k, cu, max_q=40, max_k=40))
assert torch.equal(got, c.attn(q1, lens)) and int(ev["n_freed"]) == 1 and abs(float(acc.sum()) - 2) < 1e-5
print("captured")
"""
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


@pytest.mark.gpu
def test_two_calls_at_once():
    a = [x.cuda() for x in _make([900], [900], 4, 2, 128, torch.bfloat16, 41)]
    b = [x.cuda() for x in _make([3], [9000], 7, 1, 64, torch.float16, 42)]
    cu = [_cu([900]), _cu([3]), _cu([9000])]
    call_a = lambda **kw: binding.qevict_prompt_attn(*a, cu[0], max_q=900, max_k=900, **kw)  # noqa: E731
    call_b = lambda **kw: binding.qevict_prompt_attn(*b, cu[1], cu[2], max_q=3, max_k=9000, **kw)  # noqa: E731
    want_a, want_b = call_a(), call_b()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    got_a, got_b = [], []
    for _ in range(10):
        got_a.append(call_a(stream=one))
        got_b.append(call_b(stream=two))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want_a) for x in got_a) and all(torch.equal(x, want_b) for x in got_b)


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    nq = [200, 65]
    q, k, v = (x.cuda() for x in _make(nq, nq, 4, 2, 128, torch.bfloat16, 17))
    cu = _cu(nq)
    want = binding.qevict_prompt_attn(q, k, v, cu, max_q=200, max_k=200)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.qevict_prompt_attn(q, k, v, cu, max_q=200, max_k=200, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph):
        binding.qevict_prompt_attn(q, k, v, cu, max_q=200, max_k=200, out=out)
    for lens in ([200, 65], [31, 200]):  # the lengths are read when the graph runs
        cu.copy_(_cu(lens))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        a = 0
        for x in lens:
            ro, _, spread, reach = oracle.attention(_np(q[a:a + x]), _np(k[a:a + x]), _np(v[a:a + x]))
            tol = oracle.out_tolerance(ro, spread, 6.0, x, 128, reach, 2.0 ** -8, 2.0 ** -8)
            assert (np.abs(_np(out[a:a + x]) - ro) <= tol).all()
            a += x
        assert (out[a:] == 0).all()


@pytest.mark.gpu
def test_bindings_refuse_what_the_library_cannot_see():
    q, k, v = (x.cuda() for x in _make([8], [8], 2, 1, 64, torch.float16, 1))
    cu = _cu([8])
    for call in (lambda: binding.qevict_prompt_attn(q.float(), k.float(), v.float(), cu), lambda: binding.qevict_prompt_attn(q, k, v),
                 lambda: binding.qevict_prompt_attn(q, k.to(torch.bfloat16), v, cu), lambda: binding.qevict_prompt_attn(q, k, v[:4], cu),
                 lambda: binding.qevict_prompt_attn(q, k, v, cu.long()), lambda: binding.qevict_prompt_attn(q, k, v, cu, cu[:1]),
                 lambda: binding.qevict_prompt_attn(q[..., ::2], k[..., ::2], v[..., ::2], cu), lambda: binding.qevict_prompt_attn(q.cpu(), k, v, cu),
                 lambda: binding.qevict_prompt_attn(q[..., 1:], k[..., 1:], v[..., 1:], cu)):
        with pytest.raises(binding.QEvictError):
            call()
