"""The host's arithmetic on the sizes of the attention of pieces, under UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANG = "/opt/rocm/lib/llvm/bin/clang"
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC) or not os.path.exists(CLANG), reason="needs hipcc")


def test_no_size_leaves_64_bits(tmp_path):
    from paper_2508_18224_amd.build import FLAGS
    lib, exe = tmp_path / "libchunk_san.so", tmp_path / "host_chunk_sizes_sanitize"
    src = [os.path.join(ROOT, "paper_2508_18224_amd", "csrc", s + ".hip") for s in ("cache_chunk", "profile")]
    san = ["-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined", "-g"]
    res = subprocess.run([HIPCC, *FLAGS, *san, "-o", str(lib), *src], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([CLANG, "-g", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", os.path.join(ROOT, "tests", "host_chunk_sizes_sanitize.c"), "-o", str(exe), str(lib),
                          f"-Wl,-rpath,{tmp_path}"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and run.stdout.startswith("ok "), (run.stdout + run.stderr)[-4000:]
