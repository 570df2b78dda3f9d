"""Host code of the 4-bit cache, of pages and of a context's streams on the CPU, under
AddressSanitizer + UndefinedBehaviorSanitizer, with HIP calls that work on host memory
(tests/sanitize/fake_hip.h):

* stream_checks.cpp: the books of a whole context's streams (pages, lengths, tables), in any order of
  calls and with launches that fail;
* kv_checks.cpp: what the calls on a cache refuse, and that their launches cover what they are given.
"""
import os
import subprocess

import pytest

from test_host_sanitize import B, CLANGXX, CXX_SAN, HOST_SAN, INC, ROOT, _run

pytestmark = pytest.mark.skipif(not (os.path.exists(B.HIPCC) and os.path.exists(CLANGXX)), reason="ROCm toolchain not present")
SANITIZED = ("runtime.hip", "k_pages.hip", "kv_ops.hip", "k_kv4.hip")
DRIVERS = ("stream_checks", "kv_checks")


@pytest.fixture(scope="module")
def drivers(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("san")
    objs, jobs = [], []
    for src in B.SOURCES:
        if src == "router.cpp":
            continue
        o = os.path.join(B.BUILD, os.path.splitext(src)[0] + ".o")
        san = src in SANITIZED
        if san or not (os.path.exists(o) and os.path.getmtime(o) >= os.path.getmtime(os.path.join(B.CSRC, src))):
            o = str(tmp / (os.path.splitext(src)[0] + ".o"))
            jobs.append([B.HIPCC] + B.FLAGS + (["-O1", "-g"] + HOST_SAN if san else []) + ["-c", os.path.join(B.CSRC, src), "-o", o])
        objs.append(o)
    for d in DRIVERS:
        jobs.append([CLANGXX, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include"] + CXX_SAN + INC +
                    ["-c", os.path.join(ROOT, "tests", "sanitize", d + ".cpp"), "-o", str(tmp / (d + ".o"))])
    procs = [subprocess.Popen(j, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for j in jobs]
    for j, p in zip(jobs, procs):
        out = p.communicate()[0]
        assert p.returncode == 0, " ".join(j) + "\n" + out[-4000:]
    for d in DRIVERS:
        _run([CLANGXX] + CXX_SAN + [str(tmp / (d + ".o"))] + objs +
             ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", str(tmp / d)])
    return tmp


@pytest.mark.parametrize("driver,says", [("stream_checks", "stream checks passed"), ("kv_checks", "cache checks passed")])
def test_under_asan_ubsan(drivers, driver, says):
    # (The contexts are of the library's general kernels, steps not replayed from graphs.)
    env = dict(os.environ, HH_GRAPHS="0", HH_STEP_KERNEL="0", ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(drivers / driver)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert r.returncode == 0 and says in r.stdout, r.stdout[-6000:]
    assert "runtime error" not in r.stdout and "ERROR: AddressSanitizer" not in r.stdout, r.stdout[-6000:]
