"""The cache and its attention under the checked build (see test_gpu_debug_bounds.py): the small cases pass with a clean status, and a launch whose Y is declared
shorter than it is reports LQER_ERR_BOUNDS and leaves what lies beyond untouched."""
import os
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(args, timeout=900):
    env = dict(os.environ, LQER_DEBUG_BOUNDS="1", PYTHONPATH=os.path.join(ROOT, "tests"))
    return subprocess.run([sys.executable, *args], cwd=ROOT, env=env, capture_output=True, text=True, timeout=timeout)


def test_small_cases_pass_under_the_checked_build():
    r = _run(["-m", "pytest", "-x", "-q", "-m", "gpu", "tests/test_gpu_cache.py", "tests/test_gpu_attention.py", "-k", "not 40-2-64 and not 16-1-64"])
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout


def test_a_short_extent_is_reported_and_nothing_beyond_it_is_written():
    code = textwrap.dedent("""
        import torch
        import paper_2402_02446_b200 as L
        from cache_model import Batch
        from paper_2402_02446_b200 import binding
        assert binding.DEBUG_BOUNDS and L.lib_path().endswith("liblqer_dbg.so")
        E = binding.STATUS_NAMES.index
        # a row by one CTA, a row by several, a warp a row, tiles of rows (bf16 and MXINT8), tiles divided over their keys
        for requests, dtype in (([(20, 1), (30, 1)], torch.bfloat16), ([(20, 1), (3000, 1)], torch.bfloat16), ([(9, 1)] * 1400, torch.bfloat16),
                                ([(20, 200), (30, 250)], torch.bfloat16), ([(20, 200), (30, 250)], L.MXINT8), ([(20, 40), (4000, 600)], torch.bfloat16)):
            b = Batch(requests, 16, 8, 64, 16, dtype)
            good = L.paged_attention(b.Q, b.cache, b.pages, b.step)
            assert L.poll_status(b.step.buf) == 0
            cut = 2 * 64 * 3                                  # the last three heads of the last token
            Y = torch.full_like(good, 7.0)
            L.debug_bounds_shrink(cut)
            L.paged_attention(b.Q, b.cache, b.pages, b.step, Y=Y)
            L.debug_bounds_shrink(0)
            assert L.poll_status(b.step.buf) == E("LQER_ERR_BOUNDS"), requests[:2]
            assert torch.equal(Y.flatten()[:-192], good.flatten()[:-192]) and torch.all(Y.flatten()[-192:] == 7)
            b.step.buf[:16].zero_()
            assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step), good) and L.poll_status(b.step.buf) == 0
        print("fine")
    """)
    r = _run(["-c", code])
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout[-2000:] + r.stderr[-3000:]
