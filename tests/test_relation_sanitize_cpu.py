"""The relation head's host code under AddressSanitizer and UndefinedBehaviorSanitizer
(gcc, CPU only).

relation_api.hip (argument checks, the split of the work, workspace layout) is compiled for the
host with launchers that check what the kernels take for granted and do nothing, and a child
Python runs the ABI's tests, the valid calls among them, against that build.
"""
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def test_relation_host_code_under_sanitizers(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("gcc not available")
    sys.path.insert(0, os.path.join(HERE, "sanitize"))
    import san_build as S
    sources = []
    for name in ("api", "relation_api"):
        sources.append(str(tmp_path / (name + ".cpp")))
        shutil.copyfile(os.path.join(S.CSRC, name + ".hip"), sources[-1])
    lib = str(tmp_path / "librelation_host.so")
    subprocess.check_call(["g++", "-std=c++17", *S.SAN, "-Wno-attributes", "-I" + S.HERE, "-I" + S.CSRC,
                           "-I" + os.path.join(S.ROOT, "include"), *sources, os.path.join(S.HERE, "stubs.cpp"),
                           os.path.join(HERE, "sanitize_relation", "stubs.cpp"), "-Wl,--no-undefined", "-o", lib])
    env = dict(os.environ, LD_PRELOAD=S.preload(), REX_LIBRARY=lib,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-s", "-p", "no:cacheprovider", "-m", "not gpu",
                        os.path.join(HERE, "test_relation_abi_cpu.py")],
                       env=env, cwd=str(tmp_path), capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "passed" in r.stdout and "skipped" not in r.stdout, tail
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
