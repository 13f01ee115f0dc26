"""The argument checks of the routing by scores and of the 8-bit products under host AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only, no GPU)."""
import os
import subprocess
import sys

import pytest

from test_abi_sanitized import ROOT, sanitized  # noqa: F401 (a fixture: the library with its host pass sanitized)

pytestmark = pytest.mark.slow


def test_experts_checks_run_clean_under_asan_and_ubsan(sanitized):  # noqa: F811
    _, env = sanitized
    res = subprocess.run([sys.executable, "-m", "pytest", "test_experts_abi.py", "-q", "-p", "no:cacheprovider"], env=env,
                         capture_output=True, text=True, cwd=os.path.join(ROOT, "tests"), timeout=300)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
    assert "Sanitizer" not in res.stdout + res.stderr
