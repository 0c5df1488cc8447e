"""The paged cache in the bounds-checked build."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_bounds_checked_build_passes_the_paged_cache():
    """The -DIPKV_CHECKED build compares every page's source address with the pool and every partial with the scratch, and records what lies
    outside in the status word, which these tests read after each call.  A child process, because the library variant is chosen when the
    library is first loaded."""
    env = dict(os.environ, IPKV_LIB_VARIANT="checked")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "gpu", "-x", os.path.join(ROOT, "tests", "test_paged.py"), "-k",
                        "matches_64_bits or window_and_first or bad_pages or append or keeps_what or captured"],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout.splitlines()[-1]


@pytest.mark.gpu
def test_bounds_checked_build_passes_bad_lengths_and_pages():
    env = dict(os.environ, IPKV_LIB_VARIANT="checked")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "gpu", "-x", os.path.join(ROOT, "tests", "test_paged_faults.py")],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout.splitlines()[-1]
