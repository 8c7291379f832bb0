"""The batched serving calls' host side under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): the driver tests/c_consumer/batch_stress.c against a sanitized
build of the library, over sizes up to and past the limits of the header.  No call reaches a
device."""

import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "c_consumer"))
import build_sanitized as bs  # noqa: E402


@pytest.mark.skipif(shutil.which("gcc") is None or not os.path.exists(bs.HIPCC),
                    reason="needs hipcc and a host toolchain")
def test_batch_calls_clean_under_asan_ubsan(tmp_path):
    out = str(tmp_path)
    bs.build(out)
    exe, rt = os.path.join(out, "batch_stress"), bs._asan_rt_dir()
    bs._run([bs.CLANG, "-std=c11", "-O1", "-g", "-Wall", "-Wextra", "-Werror", "-pedantic",
             "-shared-libasan", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
             "-D__HIP_PLATFORM_AMD__", "-isystem", os.path.join(bs.ROCM, "include"),
             f"-I{bs.INCLUDE}", os.path.join(bs.HERE, "batch_stress.c"), "-o", exe, "-L", out,
             "-lrelaxkv", "-Wl,-rpath," + out, "-Wl,-rpath," + rt, "-L",
             os.path.join(bs.ROCM, "lib"), "-lamdhip64",
             "-Wl,-rpath," + os.path.join(bs.ROCM, "lib"), "-lm"])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert r.stdout.startswith("ok "), r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
