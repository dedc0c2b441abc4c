"""The host side of reserved tokens, drafts and truncation under
AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: store.cpp is
compiled by g++ with both and linked to the product library for the kernels'
launchers (which a metadata-only store never calls), and the metadata-only
tests run against it in a fresh interpreter."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RUNNER = r"""
import sys
import paper_2602_22603_amd.sq as s
s.LIB_PATH = sys.argv[1]
s.lib()
maps = open("/proc/self/maps").read()
assert sys.argv[1] in maps and "libasan" in maps and "libubsan" in maps
import pytest
sys.exit(pytest.main(["-x", "-q", "-p", "no:cacheprovider", "-m", "not gpu", "tests/test_draft_host.py"]))
"""


@pytest.mark.timeout(300)
def test_draft_host_under_asan_and_ubsan(tmp_path):
    from paper_2602_22603_amd import build_lib
    try:
        runtimes = build_lib.sanitizer_runtimes()
    except RuntimeError as err:
        pytest.skip(str(err))
    if not os.path.exists(build_lib.LIB_PATH):
        build_lib.build()
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build_lib._hipcc())))
    path = str(tmp_path / "libsq_host_san.so")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(rocm, "include"), "-I", build_lib.INCLUDE, *build_lib.SAN_FLAGS,
           os.path.join(build_lib.CSRC, "store.cpp"), build_lib.LIB_PATH, "-o", path,
           f"-Wl,-rpath,{os.path.dirname(build_lib.LIB_PATH)}", "-L", os.path.join(rocm, "lib"), "-lamdhip64",
           f"-Wl,-rpath,{os.path.join(rocm, 'lib')}", "-Wl,-Bsymbolic"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, LD_PRELOAD=":".join(runtimes), ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([sys.executable, "-c", RUNNER, path], cwd=ROOT, env=env, capture_output=True,
                         text=True, timeout=240)
    tail = (res.stdout + res.stderr)[-4000:]
    assert res.returncode == 0, tail
    assert "ERROR: AddressSanitizer" not in tail and "runtime error" not in tail, tail
    assert " passed" in res.stdout, tail
