"""The 4-bit attention in the bounds-checked build."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_bounds_checked_build_passes_the_attention_over_4_bits():
    """The -DIPKV_CHECKED build compares every tile's source address with its run's extent and every partial with the scratch, and
    records what lies outside in the status word, which these tests read after each call.  A child process, because the library variant is
    chosen when the library is first loaded."""
    env = dict(os.environ, IPKV_LIB_VARIANT="checked")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-m", "gpu", "-x", os.path.join(ROOT, "tests", "test_nibble.py"),
                        os.path.join(ROOT, "tests", "test_nibble_exact.py"), "-k",
                        "matches_64_bits or shared_out or hard_values or not_a_number or 32_bits or without_tokens or within_its_own or far_out"],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout.splitlines()[-1]
