"""The host code of the rotation and paged-cache entry points under
AddressSanitizer and UndefinedBehaviorSanitizer: the boundary tests of
test_cache_host.py in a process that preloads the ASan runtime, against the
sanitized host build (as test_sanitized_host.py runs test_abi_host.py)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_cache_host_code_under_asan_and_ubsan():
    from paper_2509_24745_amd import build as B
    try:
        B.build_sanitized(verbose=False)
    except (OSError, RuntimeError) as e:
        pytest.skip(f"sanitized build unavailable: {e}")
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_cache_host.py", "-q",
                        "-p", "no:cacheprovider"], cwd=ROOT, env=B.sanitizer_env(),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "passed" in r.stdout and "failed" not in r.stdout and "skipped" not in r.stdout
