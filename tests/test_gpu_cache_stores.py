"""The stores of a step of the tables under the checked build: slots and positions that are declared shorter than they are get no entry beyond, the step
reports it, and the others are as they should be."""
import os
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_slots_beyond_a_short_extent_are_reported_and_not_written():
    code = textwrap.dedent("""
        import torch
        import paper_2402_02446_b200 as L
        from paper_2402_02446_b200 import binding
        assert binding.DEBUG_BOUNDS and L.lib_path().endswith("liblqer_dbg.so")
        E = binding.STATUS_NAMES.index
        # one launch, and two; a last row of a token and one of padding
        for added, M in (([40, 3, 20], 63), ([40, 3, 20], 70), ([3000, 7, 2000], 5007), ([3000, 7, 2000], 6000)):
            pages = L.new_page_table(3, 200, 400, 16, device="cuda:0")
            n = torch.tensor(added, dtype=torch.int32, device="cuda:0")
            good = L.cache_step(pages, n, M, commit=False)
            assert L.poll_status(good.buf) == 0
            step = L.cache_step(pages, n, M, commit=False)
            step.slots.fill_(-9)
            step.positions.fill_(-9)
            L.debug_bounds_shrink(8)
            L.cache_step(pages, n, M, step=step, commit=False)
            L.debug_bounds_shrink(0)
            assert L.poll_status(step.buf) == E("LQER_ERR_BOUNDS"), M
            for a, b in ((step.slots, good.slots), (step.positions, good.positions)):
                assert torch.equal(a[:-2], b[:-2]) and a[-2:].tolist() == [-9, -9], M
            assert torch.equal(step.lengths, good.lengths) and torch.equal(step.ring, good.ring)
            L.cache_step(pages, n, M, step=step, commit=False)
            assert L.poll_status(step.buf) == 0 and torch.equal(step.slots, good.slots)
        print("fine")
    """)
    env = dict(os.environ, LQER_DEBUG_BOUNDS="1", PYTHONPATH=os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout[-2000:] + r.stderr[-3000:]


def test_steps_and_attention_pass_under_the_checked_build():
    env = dict(os.environ, LQER_DEBUG_BOUNDS="1", PYTHONPATH=os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "tests/test_gpu_cache_step_outputs.py", "tests/test_gpu_cache_returned_entries.py",
                        "tests/test_gpu_attention_unseen.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:] + r.stderr[-2000:]
