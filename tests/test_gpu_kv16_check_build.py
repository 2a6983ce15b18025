"""Rotation and 16-bit paged cache on the checking build (-DQEVICT_DEBUG_BOUNDS), where a warp can be told to give up at one of
its waits.  The library is chosen when the binding is imported, so each part runs in a process of its own."""

import os
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code, timeout=900):
    env = dict(os.environ, QEVICT_CHECK_LIB="1", PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests")]))
    return subprocess.run([sys.executable, "-c", textwrap.dedent(code)], capture_output=True, text=True, env=env, cwd=ROOT, timeout=timeout)


def test_suites_pass_whatever_the_order_of_the_work_items():
    r = _run("""
        import sys, pytest
        from paper_2608_05326_b200 import binding, build
        build.build(variant="check")
        assert binding.lib().qevict_build_flavour() == 2
        sys.exit(pytest.main(["tests/test_rotary.py", "tests/test_kv16_cache.py", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"]))
    """)
    tail = r.stdout[-1500:] + r.stderr[-1500:]
    assert r.returncode == 0, tail
    assert " passed" in r.stdout and "failed" not in r.stdout, tail


_GIVE_UP = """
    import os, time
    import numpy as np
    import torch
    from paper_2608_05326_b200 import binding, build
    build.build(variant="check")
    assert binding.lib().qevict_build_flavour() == 2

    rng = np.random.default_rng(1)
    ragged = [int(x) for x in rng.integers(20, 700, 30)]
    # equal ranges: pairs on long contexts, tiles of rows with shared keys, both in one batch; whole items
    cases = [([1, 2, 1], [90000, 40000, 700], 32, 2, 128, torch.bfloat16), (ragged, [n + 300 for n in ragged], 4, 2, 64, torch.float16),
             ([300, 1, 1], [5000, 30000, 200], 8, 2, 128, torch.float16), ([4100], [4200], 64, 64, 64, torch.bfloat16)]
    calls = []
    for nq, lens, hq, hkv, d, dtype in cases:
        g = torch.Generator().manual_seed(len(nq))
        blocks = [-(-n // 64) for n in lens]
        table = torch.full((len(nq), max(blocks)), -1, dtype=torch.int32)
        at = 0
        for s, m in enumerate(blocks):
            table[s, :m] = torch.arange(at, at + m)
            at += m
        pools = [torch.randn((at, hkv, 64, d), generator=g).to(dtype).cuda() for _ in range(2)]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache = binding.Kv16Cache(pools[0], pools[1], table.cuda(), status)
        q = torch.randn((sum(nq), hq, d), generator=g).to(dtype).cuda()
        cu = torch.tensor(np.concatenate([[0], np.cumsum(nq)]), dtype=torch.int32, device="cuda")
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")

        def call(cache=cache, status=status, q=q, cu=cu, n=n, nq=nq, lens=lens):
            status.zero_()
            out, lse = cache.attn(q, n, cu, max_q=max(nq), max_len=max(lens), out=torch.full_like(q, 3.0), return_lse=True)
            torch.cuda.synchronize()
            return out, lse, int(status)

        call()  # warm
        calls.append((call, call()))
        assert calls[-1][1][2] == 0
    gave_up = lost = 0
    for warp in (0, 5, 9, 15, 16, 17, 18):  # softmax of both query tiles and halves; products; copies; work items
        for at in (1, 2, 3, 5, 8, 14, 30):
            for call, want in calls:
                os.environ["QEVICT_CHECK_GIVE_UP"] = "%d:%d" % (warp, at)
                t = time.perf_counter()
                out, lse, status = call()
                t = time.perf_counter() - t
                del os.environ["QEVICT_CHECK_GIVE_UP"]
                assert status in (0, 5) and t < 2.0, (warp, at, status, t)
                right = (out == want[0]).all(-1) & (lse.T == want[1].T)
                gone = out.isnan().all(-1) & lse.T.isnan()
                assert (right | gone).all(), (warp, at, int((~(right | gone)).sum()), out.shape)
                assert status == 5 or bool(right.all()), (warp, at)
                gave_up, lost = gave_up + (status == 5), lost + int(gone.sum())
                out, lse, status = call()  # and the next call is none the wiser
                assert status == 0 and torch.equal(out, want[0]) and torch.equal(lse, want[1]), (warp, at)
    assert gave_up > 60 and lost > 0, (gave_up, lost)
    print("gave up", gave_up, lost)
"""


def test_a_wait_that_gives_up_leaves_results_or_not_a_number():
    """Every warp's role, at waits from the first one on: copies, products and requests in flight have to land before the
    thread block leaves, its other warps leave with it and soon, and each row and head holds its result, or not-a-number."""
    r = _run(_GIVE_UP)
    assert r.returncode == 0 and "gave up" in r.stdout, r.stdout[-1500:] + r.stderr[-3000:]


_CLUSTERS = """
    import os
    import torch
    from paper_2608_05326_b200 import binding, build
    build.build(variant="check")
    import test_kv16_cache as t

    for most in (1, 2, 4, 8):
        os.environ["QEVICT_CHECK_CLUSTER"] = str(most)
        for nq, lens, hq, hkv, d, dtype in (([1], [2048], 32, 8, 128, torch.bfloat16), ([1, 2, 1], [8000, 1, 700], 8, 2, 64, torch.float16), ([3], [16000], 4, 1, 128, torch.float16),
                                            ([4], [900], 4, 1, 128, torch.bfloat16)):
            cache, pools, table, status, q = t._case(nq, lens, hq, hkv, d, 64, dtype, 140)
            out, lse = cache.attn(q, t._i32(lens), t._cu(nq), max_q=max(nq), max_len=max(lens), return_lse=True)
            t._check_attn(out, lse, q, pools, table, lens, nq, True, dtype)
            assert int(status) == 0
            os.environ["QEVICT_CHECK_CLUSTER"] = "16"  # what a whole device holds: the same results but for their sums' order
            whole = cache.attn(q, t._i32(lens), t._cu(nq), max_q=max(nq), max_len=max(lens), return_lse=True)
            t._check_attn(whole[0], whole[1], q, pools, table, lens, nq, True, dtype)
            del os.environ["QEVICT_CHECK_CLUSTER"]  # the device's own answer
            own = cache.attn(q, t._i32(lens), t._cu(nq), max_q=max(nq), max_len=max(lens), return_lse=True)
            assert torch.equal(own[0], whole[0]) and torch.equal(own[1], whole[1])
            os.environ["QEVICT_CHECK_CLUSTER"] = str(most)
    print("clusters")
"""


def test_a_device_that_holds_no_large_clusters_takes_smaller_ones_or_ranges():
    r = _run(_CLUSTERS)
    assert r.returncode == 0 and "clusters" in r.stdout, r.stdout[-1500:] + r.stderr[-3000:]
