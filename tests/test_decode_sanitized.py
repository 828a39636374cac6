"""The host code of sdnn_decode.h (argument checks, launch arithmetic) under AddressSanitizer and
UndefinedBehaviorSanitizer: its CPU tests against the sanitizer build of the library, in a child process."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT
from test_host_sanitized import RUNNER, _asan_runtime

MODULES = ["tests/test_decode_cpu.py", "tests/test_decode_shapes.py"]


def test_decode_host_code_under_asan_and_ubsan(tmp_path):
    runtime = _asan_runtime()
    if runtime is None:
        pytest.skip("no AddressSanitizer runtime for g++ on this host")
    from paper_2101_07948_amd import build
    lib = build.build_host_sanitized(str(tmp_path / "libsdnn_host_asan.so"))
    script = tmp_path / "run.py"
    script.write_text(RUNNER.format(root=ROOT, tests=os.path.join(ROOT, "tests"), lib=lib, modules=MODULES))
    env = dict(os.environ, LD_PRELOAD=runtime, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               CXXFLAGS="-fsanitize=undefined -fno-sanitize-recover=all")
    r = subprocess.run([sys.executable, str(script)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=1200)
    assert r.returncode == 0 and "SANITIZED_RUN_RC 0" in r.stdout, (r.stdout + r.stderr)[-4000:]
