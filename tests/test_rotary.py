"""Rotary positions by themselves against a float64 evaluation, and what the call refuses."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import rotary as oracle
from paper_2608_05326_b200 import binding

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


# ---- refusals: checked before anything reaches a device --------------------------------------------------------
def _rotation(**over):
    r = binding.qevict_rotation()
    values = dict(struct_size=C.sizeof(r), n_pairs=32, n_axes=1, interleaved=0, scale=1.0)
    values.update({k: v for k, v in over.items() if k not in ("inv_freq", "axis")})
    for n, x in values.items():
        setattr(r, n, x)
    for p in range(128):
        r.inv_freq[p], r.axis[p] = 1.0, 0
    if "inv_freq" in over:
        r.inv_freq[3] = over["inv_freq"]
    if "axis" in over:
        r.axis[3] = over["axis"]
    return r


def _args(rotation=None, **over):
    a = binding.qevict_rope_args()
    values = dict(struct_size=C.sizeof(a), device=0, dtype=1, head_dim=64, n_q_heads=4, n_k_heads=2, inverse=0, reserved=0, tokens=9,
                  positions=4096, axis_stride=9, q=4096, q_out=8192, k=4096, k_out=8192)
    values.update(over)
    for n, x in values.items():
        if not n.endswith("_stride") or n == "axis_stride":
            setattr(a, n, x)
    for n in ("q_stride", "q_out_stride", "k_stride", "k_out_stride"):
        for i, x in enumerate(values.get(n, (256, 64))):
            getattr(a, n)[i] = x
    keep = rotation or _rotation()
    a.rotation = None if rotation is False else C.addressof(keep)
    return a, keep


@pytest.mark.parametrize("over,status,word", [
    (dict(struct_size=8), 1, "struct_size"), (dict(device=-1), 1, "device"), (dict(dtype=3), 1, "dtype"), (dict(inverse=2), 1, "inverse"),
    (dict(reserved=1), 1, "reserved"), (dict(n_q_heads=0), 1, "n_q_heads"), (dict(n_k_heads=-1), 1, "n_k_heads"), (dict(tokens=-1), 1, "tokens"),
    (dict(head_dim=60), 4, "head_dim"), (dict(head_dim=264), 4, "head_dim"), (dict(n_q_heads=1025), 4, "heads"), (dict(tokens=2 ** 31), 4, "tokens"),
    (dict(head_dim=56), 1, "more channels"), (dict(q=None), 1, "NULL"), (dict(q_out=None), 1, "NULL"), (dict(k=None), 1, "NULL"), (dict(k_out=None), 1, "NULL"),
    (dict(q=4104), 1, "aligned"), (dict(k_out=8200), 1, "aligned"), (dict(q_stride=(252, 64)), 1, "strides"), (dict(k_out_stride=(256, -64)), 1, "strides"),
    (dict(q_out=4096, q_out_stride=(512, 64)), 1, "its strides"), (dict(positions=None), 1, "positions"), (dict(positions=4098), 1, "positions"),
    (dict(rotation=False), 1, "rotation is NULL"),
])
def test_unusable_arguments_are_refused_with_a_reason(over, status, word):
    a, keep = _args(**over)
    with pytest.raises(binding.QEvictError) as e:
        binding._check(binding.lib().qevict_rope(C.byref(a), None))
    assert e.value.status == status and word in str(e.value)
    del keep


@pytest.mark.parametrize("over,word", [
    (dict(struct_size=4), "struct_size"), (dict(interleaved=2), "interleaved"), (dict(n_axes=0), "n_axes"), (dict(n_axes=9), "n_axes"), (dict(n_pairs=0), "n_pairs"),
    (dict(n_pairs=6), "n_pairs"), (dict(n_pairs=132), "n_pairs"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(inv_freq=float("nan")), "inv_freq"), (dict(inv_freq=17.0), "inv_freq"), (dict(axis=1), "axis"), (dict(n_axes=3, axis=3), "axis"),
])
def test_unusable_rotations_are_refused_with_a_reason(over, word):
    a, keep = _args(_rotation(**over))
    with pytest.raises(binding.QEvictError) as e:
        binding._check(binding.lib().qevict_rope(C.byref(a), None))
    assert e.value.status == 1 and word in str(e.value)
    del keep


def test_no_tokens_need_no_device():
    a, keep = _args(tokens=0, q=None, positions=None)
    assert binding.lib().qevict_rope(C.byref(a), None) == 0
    assert binding.lib().qevict_rope(None, None) == 1
    del keep


def test_rotations_of_the_binding():
    r = binding.Rotation.standard(64, 10000.0, sections=(8, 12, 12), interleaved=True, scale=1.5)
    raw = binding.qevict_rotation.from_buffer_copy(r._packed)
    assert (raw.struct_size, raw.n_pairs, raw.n_axes, raw.interleaved, raw.scale) == (C.sizeof(raw), 32, 3, 1, 1.5)
    assert list(raw.axis)[:32] == [0] * 8 + [1] * 12 + [2] * 12 and not any(list(raw.axis)[32:])
    assert np.allclose(list(raw.inv_freq)[:32], 10000.0 ** (-np.arange(32) / 32), rtol=1e-15) and not any(list(raw.inv_freq)[32:])
    assert binding.Rotation(torch.ones(8)).n_pairs == 8
    for bad in (lambda: binding.Rotation([]), lambda: binding.Rotation([1.0] * 129), lambda: binding.Rotation([1.0] * 8, axes=[0] * 7),
                lambda: binding.Rotation([1.0] * 8, axes=[8] * 8), lambda: binding.Rotation([1.0] * 8, axes=[0.5] * 8), lambda: binding.Rotation(3),
                lambda: binding.Rotation([1.0] * 8, axes=[-1] + [0] * 7), lambda: binding.Rotation(["a"]), lambda: binding.Rotation.standard(63),
                lambda: binding.Rotation.standard(64, sections=(8, 8))):
        with pytest.raises(binding.QEvictError):
            bad()
    with pytest.raises(binding.QEvictError, match="CUDA"):
        binding.qevict_rope(torch.zeros(1, 1, 64, dtype=torch.float16), torch.zeros(1, dtype=torch.int32), r)


# ---- results ---------------------------------------------------------------------------------------------------
def _np(x):
    return x.double().cpu().numpy()


def _rot(n_pairs, n_axes, interleaved, seed, scale=1.0):
    rng = np.random.default_rng(seed)
    freq = 10000.0 ** (-np.arange(n_pairs) / n_pairs)
    axes = list(rng.permutation(np.arange(n_pairs) % n_axes))
    return binding.Rotation(freq, axes=axes, interleaved=interleaved, scale=scale), dict(inv_freq=freq, axes=axes, interleaved=interleaved, scale=scale)


def _check(got, x, pos, spec, inverse=False):
    want, size = oracle.rotate(_np(x), pos, inverse=inverse, **spec)
    tol = oracle.rotate_tolerance(want, size, pos, spec["inv_freq"], HALF_STEP[x.dtype], SMALLEST[x.dtype])
    err = np.abs(_np(got) - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())
    rest = 2 * len(spec["inv_freq"])
    assert torch.equal(got[..., rest:], x[..., rest:])


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 3, 64, 777])
@pytest.mark.parametrize("dtype,d,n_pairs,interleaved,n_axes,hq,hk", [
    (torch.bfloat16, 128, 64, False, 1, 32, 8), (torch.float16, 128, 64, False, 3, 28, 4), (torch.bfloat16, 64, 16, True, 1, 8, 8), (torch.float16, 64, 32, True, 3, 4, 2),
    (torch.bfloat16, 80, 40, False, 2, 16, 16), (torch.float16, 72, 36, False, 2, 5, 0), (torch.float16, 72, 28, True, 2, 3, 1), (torch.bfloat16, 256, 128, False, 1, 2, 1),
    (torch.float16, 256, 128, True, 8, 1, 0), (torch.bfloat16, 8, 4, False, 1, 3, 1), (torch.float16, 8, 4, True, 1, 300, 0), (torch.bfloat16, 96, 24, False, 1, 7, 7),
    (torch.bfloat16, 128, 20, False, 1, 6, 2), (torch.float16, 40, 8, True, 1, 1, 1),
])
def test_against_float64(tokens, dtype, d, n_pairs, interleaved, n_axes, hq, hk):
    rotation, spec = _rot(n_pairs, n_axes, interleaved, d + n_pairs, 1.25 if n_axes == 2 else 1.0)
    rng = np.random.default_rng(tokens)
    pos = rng.integers(-200, 140000, (n_axes, tokens))
    pos[:, 0] = [0, 1, -1, 131071, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 5][:n_axes]
    g = torch.Generator().manual_seed(tokens)
    q, k = (torch.randn((tokens, h, d), generator=g).to(dtype).cuda() for h in (hq, max(hk, 1)))
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    for inverse in (False, True):
        if hk:
            oq, ok = binding.qevict_rope(q, p, rotation, k=k, inverse=inverse)
            _check(ok, k, pos, spec, inverse)
        else:
            oq = binding.qevict_rope(q, p if n_axes > 1 else p[0], rotation, inverse=inverse)
        _check(oq, q, pos, spec, inverse)


@pytest.mark.gpu
def test_small_and_large_values():
    rotation, spec = _rot(32, 1, False, 1)
    for dtype, sizes in ((torch.float16, (2.0 ** -23, 2.0 ** -15, 30000.0)), (torch.bfloat16, (2.0 ** -130, 1e-20, 1e38))):
        for size in sizes:
            x = (torch.rand((50, 2, 64), generator=torch.Generator().manual_seed(4)).double() * size).to(dtype).cuda()
            pos = np.arange(50) * 11
            got = binding.qevict_rope(x, torch.tensor(pos, dtype=torch.int32, device="cuda"), rotation)
            _check(got, x, pos, spec)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_strided_give_the_same_bits(interleaved):
    n, hq, hk, d = 333, 6, 2, 128
    rotation, _ = _rot(48, 2, interleaved, 2)
    qkv = torch.randn((n, hq + 2 * hk, d + 8), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    q, k = qkv[:, :hq, :d], qkv[:, hq:hq + hk, 8:]
    pos = torch.randint(0, 99999, (2, 2 * n), dtype=torch.int32, device="cuda")[:, 5:5 + n]
    want = binding.qevict_rope(q.contiguous(), pos.contiguous(), rotation, k=k.contiguous())
    buf = torch.full((hq, n, d), 3.0, dtype=torch.bfloat16, device="cuda")
    got = binding.qevict_rope(q, pos, rotation, k=k, out=buf.transpose(0, 1))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0].data_ptr() == buf.data_ptr()
    rest = qkv.clone()
    binding.qevict_rope(q, pos, rotation, k=k, out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    rest[:, :hq, :d], rest[:, hq:hq + hk, 8:] = want
    assert torch.equal(qkv, rest)  # and nothing else
    text = binding.qevict_rope(want[0], pos[:1].expand(2, n), rotation)  # one position on every axis
    assert torch.equal(text, binding.qevict_rope(want[0], pos[:1].repeat(2, 1), rotation))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved,scale", [(False, 1.0), (True, 1.25)])
def test_the_gradient_is_the_transposed_rotation(interleaved, scale):
    # the columns of the map by differences (it is linear: a step of 1 from 0 in every channel) against the rows of the inverse
    d, n_pairs, token = 64, 24, 4711
    rotation, spec = _rot(n_pairs, 1, interleaved, 5, scale)
    eye = torch.eye(d, dtype=torch.float16, device="cuda")[:, None]
    pos = torch.full((d,), token, dtype=torch.int32, device="cuda")
    forward = binding.qevict_rope(eye, pos, rotation)[:, 0]   # row i: image of channel i
    backward = binding.qevict_rope(eye, pos, rotation, inverse=True)[:, 0]
    assert torch.equal(forward, backward.T)
    _check(backward[:, None], eye, np.full((1, d), token), spec, inverse=True)
    g = torch.Generator().manual_seed(6)
    x, w = (torch.randn((100, 3, d), generator=g).to(torch.float16).cuda() for _ in range(2))
    p = torch.randint(0, 5000, (100,), generator=g, dtype=torch.int32).cuda()
    left = (binding.qevict_rope(x, p, rotation).double() * w.double()).sum()  # <R x, w> = <x, R^T w>
    right = (x.double() * binding.qevict_rope(w, p, rotation, inverse=True).double()).sum()
    # each output is off by at most half a step; the roundings are weighted with the other operand
    bound = 2 * 2.0 ** -10 * scale * float((x.double().norm(dim=-1) * w.double().norm(dim=-1)).sum())
    assert abs(float(left - right)) <= bound
    if scale == 1.0:
        back = binding.qevict_rope(binding.qevict_rope(x, p, rotation), p, rotation, inverse=True)
        pair = x.double().abs().amax(-1, keepdim=True)
        assert ((back.double() - x.double()).abs() <= 6 * 2.0 ** -11 * pair + 2.0 ** -20).all()


@pytest.mark.gpu
def test_captured_replayed_and_on_another_stream():
    n, d = 40, 128
    rotation, spec = _rot(64, 1, False, 7)
    q = torch.randn((n, 8, d), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.qevict_rope(q, pos, rotation, out=out)
    for add in (0, 1000):
        pos += add
        graph.replay()
        _check(out, q, pos.cpu().numpy(), spec)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.qevict_rope(q, pos, rotation, stream=side)
    side.synchronize()
    assert torch.equal(got, out)


@pytest.mark.gpu
def test_bindings_refuse_what_the_library_cannot_see():
    rotation, _ = _rot(32, 2, False, 9)
    q = torch.zeros((5, 2, 64), dtype=torch.float16, device="cuda")
    pos = torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    for bad in (lambda: binding.qevict_rope(q.float(), pos, rotation), lambda: binding.qevict_rope(q, pos.long(), rotation), lambda: binding.qevict_rope(q, pos[0], rotation),
                lambda: binding.qevict_rope(q, pos[:, :4], rotation), lambda: binding.qevict_rope(q, pos.cpu(), rotation), lambda: binding.qevict_rope(q, pos, None),
                lambda: binding.qevict_rope(q, pos, rotation, k=q.bfloat16()), lambda: binding.qevict_rope(q, pos, rotation, k=q[:4]),
                lambda: binding.qevict_rope(q, pos, rotation, out=q[:, :1]), lambda: binding.qevict_rope(q, pos, rotation, k_out=q),
                lambda: binding.qevict_rope(q.transpose(1, 2), pos, rotation), lambda: binding.qevict_rope(q[0], pos, rotation),
                lambda: binding.qevict_rope(q, pos.T.contiguous().T, rotation), lambda: binding.qevict_rope(q[..., :32], pos, rotation)):
        with pytest.raises(binding.QEvictError):
            bad()
    assert binding.qevict_rope(q[:0], pos[:, :0], rotation).shape == (0, 2, 64)


# ---- gradients -------------------------------------------------------------------------------------------------
def _leaves(tokens, hq, hk, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((tokens, h, d), generator=g).to(dtype).cuda().requires_grad_() for h in (hq, hk)]


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,dtype,d,n_pairs,interleaved,n_axes,inverse", [
    (1, torch.bfloat16, 128, 64, False, 1, False), (77, torch.float16, 64, 16, True, 1, False), (500, torch.bfloat16, 128, 40, False, 3, True), (0, torch.float16, 64, 32, False, 1, False),
])
def test_gradients_reach_queries_and_keys(tokens, dtype, d, n_pairs, interleaved, n_axes, inverse):
    rotation, spec = _rot(n_pairs, n_axes, interleaved, 21, 1.25)
    q, k = _leaves(tokens, 6, 2, d, dtype, 22)
    wq, wk = (x.detach().flip(-1) + 1 for x in (q, k))
    pos = torch.randint(0, 9999, (n_axes, tokens), generator=torch.Generator().manual_seed(23), dtype=torch.int32).cuda()
    oq, ok = binding.qevict_rope(q, pos, rotation, k=k, inverse=inverse)
    plain = binding.qevict_rope(q.detach(), pos, rotation, k=k.detach(), inverse=inverse)
    assert torch.equal(oq, plain[0]) and torch.equal(ok, plain[1]) and not plain[0].requires_grad
    torch.autograd.backward([oq, ok], [wq, wk])
    for got, w in ((q.grad, wq), (k.grad, wk)):
        _check(got, w, _np(pos), spec, not inverse)
    # one of them alone, with and without the other
    for part in (0, 1):
        q2, k2 = (x.detach().requires_grad_(i == part) for i, x in enumerate((q, k)))
        both = binding.qevict_rope(q2, pos, rotation, k=k2, inverse=inverse)
        assert [x.requires_grad for x in both] == [part == 0, part == 1]
        both[part].backward((wq, wk)[part])
        assert torch.equal((q2, k2)[part].grad, (q, k)[part].grad) and (q2, k2)[1 - part].grad is None
        alone = (q, k)[part].detach().requires_grad_()
        binding.qevict_rope(alone, pos, rotation, inverse=inverse).backward((wq, wk)[part])
        assert torch.equal(alone.grad, (q, k)[part].grad)
    # a loss that sees one of two outputs: the other has no gradient
    q3, k3 = (x.detach().requires_grad_() for x in (q, k))
    binding.qevict_rope(q3, pos, rotation, k=k3, inverse=inverse)[1].backward(wk)
    assert q3.grad is None and torch.equal(k3.grad, k.grad)


@pytest.mark.gpu
def test_gradients_by_differences_and_of_the_gradient():
    # the map is linear, so a step of any size from 0 is its derivative, but for roundings: <w, R (x + e) - R x> against <grad, e>
    rotation, spec = _rot(24, 1, False, 24)
    x = _leaves(40, 3, 1, 64, torch.float16, 25)[0]
    at = x.detach()
    pos = torch.arange(40, dtype=torch.int32, device="cuda") * 7
    w, e = (torch.randn_like(x).detach() for _ in range(2))
    (grad,) = torch.autograd.grad(binding.qevict_rope(x, pos, rotation), x, w)
    moved = binding.qevict_rope(at + e, pos, rotation).double() - binding.qevict_rope(at, pos, rotation).double()
    left, right = (w.double() * moved).sum(), (grad.double() * ((at + e).double() - at.double())).sum()
    # three roundings of at most half a step: of both images, weighted with w, and of the gradient, weighted with the step
    size = sum(float((a.double().norm(dim=-1) * b.double().norm(dim=-1)).sum()) for a, b in ((w, at + e), (w, at), (w, (at + e).double() - at.double())))
    assert abs(float(left - right)) <= 2.0 ** -11 * 2 ** 0.5 * 1.01 * size
    # gradients of gradients: <grad(w), u> as a function of w has the gradient R u
    v = w.clone().requires_grad_()
    (first,) = torch.autograd.grad(binding.qevict_rope(x, pos, rotation), x, v, create_graph=True)
    (second,) = torch.autograd.grad(first, v, e)
    assert torch.equal(second, binding.qevict_rope(e, pos, rotation))


@pytest.mark.gpu
def test_gradients_of_any_strides_and_streams():
    rotation, _ = _rot(32, 1, True, 26)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    q = _leaves(50, 4, 1, 64, torch.bfloat16, 27)[0]
    for make in (lambda y: y.sum(), lambda y: y[:, 1].sum(), lambda y: (y.transpose(0, 1).reshape(4, -1) * torch.arange(4, device="cuda", dtype=y.dtype)[:, None]).sum(),
                 lambda y: (y.transpose(1, 2) * 2).sum(), lambda y: y[..., 1:].sum()):
        (want_g,) = torch.autograd.grad(make((z := binding.qevict_rope(q.detach(), pos, rotation).requires_grad_())), z)
        want = binding.qevict_rope(want_g.contiguous(), pos, rotation, inverse=True)
        (got,) = torch.autograd.grad(make(binding.qevict_rope(q, pos, rotation)), q)
        assert torch.equal(got, want)
    wide = torch.randn((50, 4 * 64 + 4), dtype=torch.bfloat16, device="cuda")  # a gradient that starts off the 16 bytes
    off = wide[:, 4:].view(50, 4, 64)
    (got,) = torch.autograd.grad(binding.qevict_rope(q, pos, rotation), q, off)
    assert torch.equal(got, binding.qevict_rope(off.contiguous(), pos, rotation, inverse=True))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = binding.qevict_rope(q, pos, rotation, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    (got,) = torch.autograd.grad(y, q, torch.ones_like(y))
    torch.cuda.synchronize()
    assert torch.equal(got, binding.qevict_rope(torch.ones_like(q).detach(), pos, rotation, inverse=True))


@pytest.mark.gpu
def test_gradients_in_a_captured_step():
    rotation, spec = _rot(32, 1, False, 28)
    q = _leaves(60, 4, 1, 64, torch.float16, 29)[0]
    pos = torch.arange(60, dtype=torch.int32, device="cuda")
    w = torch.randn_like(q).detach()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(binding.qevict_rope(q, pos, rotation), q, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        (grad,) = torch.autograd.grad(binding.qevict_rope(q, pos, rotation), q, w)
    for _ in range(2):
        w.copy_(torch.randn_like(w))
        graph.replay()
        _check(grad, w, pos.cpu().numpy(), spec, True)


@pytest.mark.gpu
def test_a_gradient_is_not_lost_in_given_outputs():
    rotation, _ = _rot(32, 1, False, 30)
    q, k = _leaves(5, 2, 2, 64, torch.float16, 31)
    pos, plain = torch.arange(5, dtype=torch.int32, device="cuda"), q.detach()
    for bad in (lambda: binding.qevict_rope(q, pos, rotation, out=plain), lambda: binding.qevict_rope(plain, pos, rotation, k=k, k_out=plain),
                lambda: binding.qevict_rope(plain, pos, rotation, k=k, out=plain), lambda: binding.qevict_rope(plain, pos, rotation, out=q)):
        with pytest.raises(binding.QEvictError, match="gradient"):
            bad()
    with torch.no_grad():
        out = torch.empty_like(plain)
        assert binding.qevict_rope(q, pos, rotation, out=out) is out and not out.requires_grad
        assert not binding.qevict_rope(q, pos, rotation).requires_grad
    assert binding.qevict_rope(plain, pos, rotation, out=out) is out
    y = binding.qevict_rope(q, pos, rotation)
    pos += 1  # what the gradient needs is not the same any more
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
