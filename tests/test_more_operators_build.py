"""What can be seen of the rotation, the read of a cache and the attention of pieces of prompts without a GPU: their host code under AddressSanitizer and UndefinedBehaviorSanitizer
(device code is not instrumented), and the code generated for their kernels."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CSRC = os.path.join(ROOT, "paper_2508_18224_amd", "csrc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """Assembly of each source, by name."""
    from paper_2508_18224_amd.build import FLAGS
    at = tmp_path_factory.mktemp("code")
    flags = [f for f in FLAGS if f not in ("-shared", "-fPIC")]
    text = {}
    for source in ("rotary", "cache_read", "cache_chunk"):
        res = subprocess.run([HIPCC, *flags, "--offload-device-only", "-S", "-o", str(at / source), os.path.join(CSRC, source + ".hip")], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-3000:]
        text[source] = (at / source).read_text()
    return text


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    from paper_2508_18224_amd.build import FLAGS
    lib = tmp_path / "libmore_san.so"
    src = [os.path.join(CSRC, s + ".hip") for s in ("rotary", "cache_read", "cache_chunk", "profile")]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    res = subprocess.run([HIPCC, *FLAGS, *san, "-shared-libsan", "-o", str(lib), *src], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    exe = tmp_path / "host_more_operators_sanitize"
    clang = "/opt/rocm/lib/llvm/bin/clang"
    res = subprocess.run([clang, "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-shared-libsan",
                          os.path.join(ROOT, "tests", "host_more_operators_sanitize.c"), "-o", str(exe), str(lib), f"-Wl,-rpath,{tmp_path}"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    rt = subprocess.run([clang, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    if rt and os.path.exists(rt):
        env["LD_LIBRARY_PATH"] = os.path.dirname(rt) + ":" + env.get("LD_LIBRARY_PATH", "")
    run = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=600)
    assert run.returncode == 0, (run.stdout + run.stderr)[-4000:]
    assert run.stdout.startswith("ok "), run.stdout
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-4000:]


def test_a_wait_state_follows_every_write_of_m0(code):
    """Loads straight to LDS take their LDS address from m0, which needs a wait state after it is written; the compiler does not keep that distance inside assembly blocks."""
    loads, since = 0, 99
    for line in code["cache_chunk"].splitlines():
        op = line.split(";")[0].strip()
        if not op or op.startswith(".") or op.endswith(":"):
            continue
        if re.match(r"buffer_load_\w+ .*\blds\b", op):
            loads += 1
            assert since >= 1, line
        if re.match(r"s_\w+ m0\b", op):
            since = 0
        else:
            since += int(op.split()[1], 0) + 1 if op.startswith("s_nop") else 1
    assert loads >= 22                                             # two a tile: seven tiles in front of the loop, two in it, two where values are not finite


@pytest.mark.parametrize("source,kernels", [("rotary", 1), ("cache_read", 2), ("cache_chunk", 3)])
def test_everything_is_kept_in_registers(code, source, kernels):
    """A reload in the loop over the pieces would wait for the keys and values that are on their way to LDS."""
    spills = re.findall(r"\.name:\s+(_ZN3nsa\S+)\n(?:.*\n)*?\s+\.vgpr_spill_count:\s+(\d+)", code[source])
    scratch = re.findall(r"\.name:\s+(_ZN3nsa\S+)\n\s+\.private_segment_fixed_size:\s+(\d+)", code[source])
    assert len(spills) == len(scratch) == kernels and [n for _, n in spills + scratch if n != "0"] == []
