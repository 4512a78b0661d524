"""The host side of the speculative decoding calls under the host sanitizers (CPU only): the
refusals of tests/test_draft_host.py against the instrumented library."""
import glob
import os
import subprocess
import sys

import pytest
import torch

from test_host_sanitizers import HIPCC, OUT, ROOT, RUNTIME, _build


def _library():
    """The instrumented library: the one that is there if it is newer than every source."""
    lib = os.path.join(OUT, "libtailupdate_sanitized.so")
    srcs = glob.glob(os.path.join(ROOT, "paper_2609_18935_amd", "csrc", "*")) + \
        glob.glob(os.path.join(ROOT, "include", "*"))
    if os.path.exists(lib) and all(os.path.getmtime(lib) > os.path.getmtime(s) for s in srcs):
        return lib
    return _build()


@pytest.mark.skipif(torch.cuda.is_available(), reason="those tests run without a GPU")
@pytest.mark.skipif(not RUNTIME or not os.path.exists(HIPCC), reason="no hipcc or no sanitizer runtime")
def test_draft_calls_under_asan_and_ubsan():
    lib = _library()
    env = dict(os.environ)
    env.update({"LD_PRELOAD": RUNTIME[-1], "TU_LIBRARY": lib,
                "ASAN_OPTIONS": "detect_leaks=0:halt_on_error=1:abort_on_error=1",
                "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1"})
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_draft_host.py"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert r.returncode == 0, out[-4000:]
    assert " passed" in out
