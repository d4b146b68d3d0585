"""The host code of the output head's entry points (checks, plans, workspace
sizes) under AddressSanitizer and UndefinedBehaviorSanitizer: the tests of
refusals and limits run on an instrumented build of the library."""
import os
import subprocess
import sys

import pytest

from test_sanitizers_cpu import HIPCC, ROOT, _clang_asan_runtime


def test_head_host_code_under_asan_and_ubsan(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    asan = _clang_asan_runtime()
    if asan is None:
        pytest.skip("clang's AddressSanitizer runtime not found")
    from paper_2609_20359_amd import build as B

    out = str(tmp_path / "libflround_san.so")
    host_san = []
    for f in ("-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
              "-fno-omit-frame-pointer"):
        host_san += ["-Xarch_host", f]
    B.build(out=out, extra=host_san + ["-Xarch_host", "-g"])
    with open(out, "rb") as f:
        assert b"__asan_report" in f.read()   # the host code is instrumented
    env = dict(os.environ)
    env["FLROUND_LIB"] = out
    env["LD_PRELOAD"] = asan + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "not gpu",
                        "-p", "no:cacheprovider", "tests/test_head_abi_cpu.py",
                        "tests/test_head_limits_cpu.py"],
                       env=env, cwd=ROOT, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, (r.stdout[-4000:], r.stderr[-4000:])
    assert " passed" in r.stdout
