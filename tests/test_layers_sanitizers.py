"""Host code of the layers' operators under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): the refusals, tables and
workspace sizes of test_layers_cpu.py against the instrumented copy of the library."""
import glob
import os
import shutil
import subprocess
import sys

import pytest

from conftest import ROOT
from test_host_sanitizers import HIPCC, _build_module


@pytest.mark.skipif(not (shutil.which(HIPCC) or os.path.exists(HIPCC)), reason="needs hipcc to build the library")
def test_layers_host_code_is_clean_under_asan_and_ubsan():
    b = _build_module()
    sources = glob.glob(os.path.join(b.CSRC, "*")) + glob.glob(os.path.join(b.INCLUDE, "*")) + [b.__file__]
    lib = b.SANITIZE_LIB
    if not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(s) for s in sources):
        lib = b.build(verbose=False, sanitize=True)
    env = dict(os.environ)
    env.update({"LD_PRELOAD": b.sanitizer_runtime(), "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
                "UBSAN_OPTIONS": "print_stacktrace=1:halt_on_error=1", "ROLLOUT_LIBRARY": lib})
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "tests/test_layers_cpu.py"],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = res.stdout[-3000:] + res.stderr[-3000:]
    assert res.returncode == 0, out
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out
    assert " passed" in res.stdout
