"""The host side of the operators in include/fluxbin_serve.h under AddressSanitizer and UndefinedBehaviorSanitizer, as
test_host_sanitizers.py runs that of include/fluxbin.h."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_serve_host_tests_pass_under_asan_and_ubsan(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2608_15602_amd import build as b
    try:
        b.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    lib = b.build_host_sanitized(verbose=False)
    rt = b.asan_runtime()
    assert os.path.exists(rt), rt
    log = tmp_path / "san"
    env = dict(os.environ)
    env.update(LD_PRELOAD=rt, FLUXBIN_LIBRARY=lib,
               ASAN_OPTIONS=f"detect_leaks=0:abort_on_error=1:log_path={log}",
               UBSAN_OPTIONS=f"halt_on_error=1:print_stacktrace=1:log_path={log}")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_serve_host.py"), "-q", "-x",
                        "-k", "not binding", "-p", "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=600)
    reports = "".join(p.read_text() for p in tmp_path.glob("san*"))
    assert r.returncode == 0 and not reports, (r.stdout[-3000:], r.stderr[-3000:], reports[:5000])
