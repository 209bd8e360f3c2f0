"""The dense-document ABI checks under the host sanitizers: a child interpreter with
the sanitizer runtime preloaded runs tests/test_dense_abi.py on the sanitized
library."""

import os
import subprocess
import sys

import pytest

from conftest import ROOT


def test_dense_abi_checks_pass_under_the_sanitizers():
    hostsan = pytest.importorskip("paper_2609_05138_amd.build_hostsan")
    try:
        hostsan.asan_runtime()
    except RuntimeError as e:
        pytest.skip(str(e))
    hostsan.build()
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_dense_abi.py")],
                       capture_output=True, text=True, env=hostsan.runtime_env(), cwd=ROOT, timeout=600)
    out = r.stdout + r.stderr
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0 and " passed" in r.stdout, out[-6000:]
