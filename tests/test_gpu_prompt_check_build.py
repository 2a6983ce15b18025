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
