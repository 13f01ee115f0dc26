"""The training operators' argument checks under host AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only, no GPU)."""
import os
import subprocess
import sys

import pytest

from test_abi_sanitized import ROOT, sanitized  # noqa: F401 (a fixture: the library with its host pass sanitized)

pytestmark = pytest.mark.slow


def test_training_checks_run_clean_under_asan_and_ubsan(sanitized):  # noqa: F811
    _, env = sanitized
    res = subprocess.run([sys.executable, "-m", "pytest", "test_train_abi.py", "test_train_refusals.py", "-q",
                          "-p", "no:cacheprovider"], env=env, capture_output=True, text=True, cwd=os.path.join(ROOT, "tests"),
                         timeout=300)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
    assert "Sanitizer" not in res.stdout + res.stderr
