"""The calls on pages and drafted trees under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only):
their argument checks, workspace sizes and the fault-injection path, as test_sanitized_host does for the rest."""
import glob
import os
import subprocess
import sys

import pytest

from paper_2608_14498_amd import build as rbuild
from tests.test_sanitized_host import ROOT, _asan_runtime, _stale


def test_pages_and_trees_pass_under_asan_and_ubsan(tmp_path):
    rt = _asan_runtime()
    if rt is None or not os.path.exists(rbuild.HIPCC):
        pytest.skip("no hipcc or clang ASan runtime in this image")
    if _stale(rbuild.ASAN_LIB):
        rbuild.build(sanitize=True)
    log = str(tmp_path / "san")
    env = dict(os.environ, RP_LIBRARY=rbuild.ASAN_LIB, LD_PRELOAD=rt,
               ASAN_OPTIONS=f"detect_leaks=0:abort_on_error=1:log_path={log}",
               UBSAN_OPTIONS=f"halt_on_error=1:print_stacktrace=1:log_path={log}")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_pages_cpu.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    reports = "".join(open(p).read() for p in glob.glob(log + "*"))
    assert r.returncode == 0 and not reports, (r.stdout[-3000:] + r.stderr[-3000:] + reports[:6000])
    assert "passed" in r.stdout
