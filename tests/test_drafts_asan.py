"""The host checks of include/delta_drafts.h (tests/test_drafts_cpu.py) once more, against a build of the
library whose C ABI sources are compiled with AddressSanitizer; the kernels are the release build's."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2510_09883_amd")
API = ["delta_api", "extend_api", "drafts_api"]


def test_drafts_cpu_tests_pass_with_host_address_sanitizer(tmp_path):
    from paper_2510_09883_amd import build as B
    gxx = shutil.which("g++")
    objs = [os.path.join(PKG, "_build", s.rsplit(".", 1)[0] + ".o") for s in B.SOURCES if s.rsplit(".", 1)[0] not in API]
    if gxx is None or not all(os.path.exists(o) for o in objs):
        pytest.skip("needs g++ and the release build's kernel objects (run the build first)")
    api = []
    for src in API:
        api.append(str(tmp_path / (src + ".o")))
        subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fPIC", "-fsanitize=address", "-fno-omit-frame-pointer",
                        "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-c",
                        os.path.join(PKG, "csrc", src + ".cpp"), "-o", api[-1]], check=True)
    lib = str(tmp_path / "libdelta_attn_asan.so")
    subprocess.run([gxx, "-shared", "-fsanitize=address", *objs, *api, "-L/opt/rocm/lib", "-lamdhip64", "-o", lib],
                   check=True)
    libasan = subprocess.run([gxx, "-print-file-name=libasan.so"], capture_output=True, text=True,
                             check=True).stdout.strip()
    env = dict(os.environ, LD_PRELOAD=libasan, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", DELTA_ATTN_LIB=lib)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_drafts_cpu.py")], env=env, capture_output=True, text=True,
                       timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "AddressSanitizer" not in r.stderr
