"""Prompt attention and the 8-bit cache on the checking build (-DQEVICT_DEBUG_BOUNDS), in which the prompt kernel's work
items come in falling order.  The library is chosen when the binding is imported, so each part runs in a process of its own."""

import os
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code, extra_env=None, timeout=900):
    env = dict(os.environ, QEVICT_CHECK_LIB="1", PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests")]))
    env.update(extra_env or {})
    return subprocess.run([sys.executable, "-c", textwrap.dedent(code)], capture_output=True, text=True, env=env,
                          cwd=ROOT, timeout=timeout)


def test_suites_pass_whatever_the_order_of_the_work_items():
    r = _run("""
        import sys, pytest
        from paper_2608_05326_b200 import binding, build
        build.build(variant="check")
        assert binding.lib().qevict_build_flavour() == 2
        sys.exit(pytest.main(["tests/test_prompt_attn.py", "tests/test_kv8_cache.py", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"]))
    """)
    tail = r.stdout[-1500:] + r.stderr[-1500:]
    assert r.returncode == 0, tail
    assert " passed" in r.stdout and "failed" not in r.stdout, tail


_CALLS = """
    import os, time
    import numpy as np
    import torch
    from paper_2608_05326_b200 import binding, build
    build.build(variant="check")
    assert binding.lib().qevict_build_flavour() == 2

    def cu(lens):
        return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")

    rng = np.random.default_rng(1)
    ragged = [int(x) for x in rng.integers(1, 700, 40)]
    # several work items for every SM; one or two tiles of keys each; keys split over thread blocks
    cases = [(ragged, ragged, 8, 2, 128, torch.bfloat16), ([150] * 200, [150] * 200, 3, 3, 64, torch.float16), ([2, 40], [9000, 6001], 4, 2, 128, torch.float16)]
    calls = []
    for nq, nk, hq, hkv, d, dtype in cases:
        g = torch.Generator().manual_seed(len(nq))
        q, k, v = (torch.randn((sum(n), h, d), generator=g).to(dtype).cuda() for n, h in ((nq, hq), (nk, hkv), (nk, hkv)))
        bounds = cu(nq), cu(nk)

        def call(q=q, k=k, v=v, bounds=bounds, nq=nq, nk=nk):
            out, lse = torch.full_like(q, 3.0), torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            binding.qevict_prompt_attn(q, k, v, *bounds, max(nq), max(nk), out=out, lse=lse, status=status)
            torch.cuda.synchronize()
            return out, lse, int(status)

        call()  # warm
        calls.append((call, call()))
        assert calls[-1][1][2] == 0
"""

_GIVE_UP = _CALLS + """
    gave_up = 0
    for warp in (0, 5, 9, 15, 16, 17, 18):  # softmax of both query tiles and halves; products; copies; work items
        for at in (1, 2, 3, 4, 7, 12, 30):
            for call, want in calls:
                os.environ["QEVICT_CHECK_GIVE_UP"] = "%d:%d" % (warp, at)
                t = time.perf_counter()
                out, lse, status = call()
                t = time.perf_counter() - t
                del os.environ["QEVICT_CHECK_GIVE_UP"]
                assert status in (0, 5) and t < 2.0, (warp, at, status, t)
                gave_up += status == 5
                if status == 0:  # no CTA comes to that wait
                    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
                out, lse, status = call()  # and the next call is none the wiser
                assert status == 0 and torch.equal(out, want[0]) and torch.equal(lse, want[1]), (warp, at)
    assert gave_up > 60, gave_up
    print("gave up", gave_up)
"""


def test_a_wait_that_gives_up_ends_the_call_with_a_status():
    """Every warp's role, at waits from the first one on: copies, products and requests in flight have to land before the
    thread block leaves, its other warps have to leave with it and soon."""
    r = _run(_GIVE_UP)
    assert r.returncode == 0 and "gave up" in r.stdout, r.stdout[-1500:] + r.stderr[-3000:]


_ROWS = _CALLS + """
    lost = rows = 0
    for warp in (0, 6, 11, 15, 16, 17, 18):
        for at in (1, 2, 3, 5, 6, 8, 10, 14, 20):
            for call, want in calls:
                os.environ["QEVICT_CHECK_GIVE_UP"] = "%d:%d" % (warp, at)
                out, lse, status = call()
                del os.environ["QEVICT_CHECK_GIVE_UP"]
                right = (out == want[0]).all(-1) & (lse.T == want[1].T)
                gone = out.isnan().all(-1) & lse.T.isnan()
                assert (right | gone).all(), (warp, at, int((~(right | gone)).sum()), out.shape)
                assert status == (5 if gone.any() else 0) or bool(right.all()), (warp, at, status)
                lost, rows = lost + int(gone.sum()), rows + gone.numel()
    assert 0 < lost < rows
    print("lost", lost, rows)
"""


def test_a_row_without_a_result_is_not_a_number():
    """Whatever a call has to give up: each row and head holds its result, or not-a-number in every channel and in lse."""
    r = _run(_ROWS)
    assert r.returncode == 0 and "lost" in r.stdout, r.stdout[-1500:] + r.stderr[-3000:]
