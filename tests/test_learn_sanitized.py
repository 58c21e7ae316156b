"""The learner's argument checks under AddressSanitizer and UndefinedBehaviorSanitizer (CPU
only): tests/sanitize/learn_host_checks.hip compiles csrc/learn.hip in, instrumented on the
host pass, and makes every call that has to be refused before any device work."""
import os
import subprocess

import pytest

from paper_2207_07736_amd import build

ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
CLANG = os.path.join(ROCM, "llvm", "bin", "clang++")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(not (os.path.exists(build.HIPCC) and os.path.exists(CLANG)), reason="needs hipcc and clang")


def test_refusals_under_asan_and_ubsan(tmp_path):
    obj, exe = tmp_path / "learn_host_checks.o", tmp_path / "learn_host_checks"
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-Xarch_host", "-g"]
    flags = [f for f in build.FLAGS if f not in ("-O3", "-shared", "-fPIC")] + ["-O1"]
    subprocess.run([build.HIPCC, *flags, *san, "-I", build.INCLUDE, "-c", "-o", str(obj),
                    os.path.join(ROOT, "tests", "sanitize", "learn_host_checks.hip")], check=True, capture_output=True, text=True)
    subprocess.run([CLANG, "-fsanitize=address,undefined", "-o", str(exe), str(obj), "-L", os.path.join(ROCM, "lib"),
                    "-lamdhip64", f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}"], check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    out = res.stdout + res.stderr
    assert res.returncode == 0 and "learn host checks: OK" in res.stdout, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out
