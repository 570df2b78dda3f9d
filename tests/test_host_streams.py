"""The books of a context's streams (pages, lengths, tables) on the CPU, under AddressSanitizer +
UndefinedBehaviorSanitizer: tests/sanitize/stream_checks.cpp drives a whole context whose
HIP calls work on host memory, in any order of calls and with launches that fail."""
import os
import subprocess

import pytest

from test_host_sanitize import B, CLANGXX, CXX_SAN, HOST_SAN, INC, ROOT, _run


@pytest.mark.skipif(not (os.path.exists(B.HIPCC) and os.path.exists(CLANGXX)), reason="ROCm toolchain not present")
def test_streams_under_asan_ubsan(tmp_path):
    objs, jobs = [], []
    for src in B.SOURCES:
        if src in ("kv_ops.hip", "router.cpp"):
            continue
        o = os.path.join(B.BUILD, os.path.splitext(src)[0] + ".o")
        san = src in ("runtime.hip", "k_pages.hip")
        if san or not (os.path.exists(o) and os.path.getmtime(o) >= os.path.getmtime(os.path.join(B.CSRC, src))):
            o = str(tmp_path / (os.path.splitext(src)[0] + ".o"))
            jobs.append([B.HIPCC] + B.FLAGS + (["-O1", "-g"] + HOST_SAN if san else []) + ["-c", os.path.join(B.CSRC, src), "-o", o])
        objs.append(o)
    driver = str(tmp_path / "stream_checks.o")
    jobs.append([CLANGXX, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include"] + CXX_SAN + INC +
                ["-c", os.path.join(ROOT, "tests", "sanitize", "stream_checks.cpp"), "-o", driver])
    procs = [subprocess.Popen(j, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for j in jobs]
    for j, p in zip(jobs, procs):
        out = p.communicate()[0]
        assert p.returncode == 0, " ".join(j) + "\n" + out[-4000:]
    exe = str(tmp_path / "stream_checks")
    _run([CLANGXX] + CXX_SAN + [driver] + objs + ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    # (The contexts are of the library's general kernels, steps not replayed from graphs.)
    env = dict(os.environ, HH_GRAPHS="0", HH_STEP_KERNEL="0", ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "stream checks passed" in r.stdout, r.stdout[-6000:]
    assert "runtime error" not in r.stdout and "ERROR: AddressSanitizer" not in r.stdout, r.stdout[-6000:]
