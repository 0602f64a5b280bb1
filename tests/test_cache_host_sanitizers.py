"""The host code of the calls over a paged cache (checks, how a call is cut, workspace sizes) under AddressSanitizer and UndefinedBehaviorSanitizer, driven
by a C program over shapes at the limits.  Device code is not instrumented and no GPU is involved."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCES = ["cache_api.hip", "cache_append.hip", "cache_attend.hip", "select.hip", "profile.hip"]


@pytest.mark.skipif(not os.path.exists(HIPCC) or shutil.which("gcc") is None, reason="needs hipcc and gcc")
def test_host_code_of_the_cache_is_clean_under_asan_and_ubsan(tmp_path):
    from paper_2508_18224_amd.build import FLAGS
    lib = tmp_path / "libcache_san.so"
    src = [os.path.join(ROOT, "paper_2508_18224_amd", "csrc", s) for s in SOURCES]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    res = subprocess.run([HIPCC, *FLAGS, *san, "-shared-libsan", "-o", str(lib), *src], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    exe = tmp_path / "host_cache_sanitize"
    clang = "/opt/rocm/lib/llvm/bin/clang"
    res = subprocess.run([clang, "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-shared-libsan",
                          os.path.join(ROOT, "tests", "host_cache_sanitize.c"), "-o", str(exe), str(lib),
                          f"-Wl,-rpath,{tmp_path}"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    rt = subprocess.run([clang, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    if rt and os.path.exists(rt):
        env["LD_LIBRARY_PATH"] = os.path.dirname(rt) + ":" + env.get("LD_LIBRARY_PATH", "")
    run = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=600)
    assert run.returncode == 0, (run.stdout + run.stderr)[-4000:]
    assert run.stdout.startswith("ok "), run.stdout
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-4000:]
