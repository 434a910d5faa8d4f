"""The validation layer of the paging entry points (csrc/paging_api.cpp)
under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: built for
the host with g++ and host stand-ins for the launchers, and put through
tests/test_paging_abi.py in a child process."""

import os
import shutil
import subprocess
import sys
import tempfile

import pytest

from tests.test_abi_sanitized import ROCM, ROOT, _libasan


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "lib", "libamdhip64.so")),
                    reason="needs g++ and the HIP runtime library")
def test_paging_validation_under_asan_ubsan():
    asan = _libasan()
    if asan is None:
        pytest.skip("no libasan for g++")
    tmp = tempfile.mkdtemp(prefix="nvfp4_san_")
    try:
        so = os.path.join(tmp, "libnvfp4_san.so")
        csrc, stubs = os.path.join(ROOT, "paper_2609_04098_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize")
        cmd = ["g++", "-std=c++17", "-O1", "-g", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
               "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", csrc,
               "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
               os.path.join(csrc, "api.cpp"), os.path.join(csrc, "attention_api.cpp"), os.path.join(csrc, "paging_api.cpp"),
               os.path.join(stubs, "launch_stubs.cpp"), os.path.join(stubs, "attention_launch_stubs.cpp"),
               os.path.join(stubs, "paging_launch_stubs.cpp"),
               "-L", os.path.join(ROCM, "lib"), "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-lamdhip64", "-o", so]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        code = ("import sys; sys.path.insert(0, %r); "
                "import paper_2609_04098_amd.nvfp4 as C; C.LIB_PATH = %r; "
                "import pytest; sys.exit(pytest.main(['-q', '-p', 'no:cacheprovider', %r]))"
                % (ROOT, so, os.path.join(ROOT, "tests", "test_paging_abi.py")))
        logs = os.path.join(tmp, "report")
        env = dict(os.environ, LD_PRELOAD=asan, PYTHONDONTWRITEBYTECODE="1", PYTHONMALLOC="malloc",
                   HIP_VISIBLE_DEVICES="",
                   ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:exitcode=97:log_path=" + logs,
                   UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1:exitcode=98:log_path=" + logs)
        r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True,
                           timeout=600)
        reports = [os.path.join(tmp, f) for f in os.listdir(tmp) if f.startswith("report")]
        text = "".join(open(f).read() for f in reports)
        assert not reports, text[:4000]
        assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
        assert " passed" in r.stdout
    finally:
        shutil.rmtree(tmp, ignore_errors=True)
