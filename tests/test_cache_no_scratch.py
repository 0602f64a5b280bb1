"""The kernels over a paged cache keep whole pieces and pages in registers: none may spill, and the buffers of the attention must be
scalar (where the compiler cannot see that it wraps every load in a loop over the lanes)."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _code(tmp_path, source):
    from paper_2508_18224_amd.build import FLAGS
    out = tmp_path / "out.s"
    flags = [f for f in FLAGS if f not in ("-shared", "-fPIC")]
    res = subprocess.run([HIPCC, *flags, "--offload-device-only", "-S", "-o", str(out),
                          os.path.join(ROOT, "paper_2508_18224_amd", "csrc", source)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return out.read_text()


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("source,kernels", [("cache_attend.hip", 17), ("cache_append.hip", 9)])
def test_no_kernel_spills_vector_registers(tmp_path, source, kernels):
    text = _code(tmp_path, source)
    spills = dict(re.findall(r"\.name:\s+(_ZN3nsa\S+)\n(?:.*\n)*?\s+\.vgpr_spill_count:\s+(\d+)", text))
    scratch = dict(re.findall(r"\.name:\s+(_ZN3nsa\S+)\n\s+\.private_segment_fixed_size:\s+(\d+)", text))
    assert len(spills) >= kernels and scratch.keys() == spills.keys(), sorted(spills)
    assert {k: (n, scratch[k]) for k, n in spills.items() if n != "0" or scratch[k] != "0"} == {}
    if source == "cache_attend.hip":
        loads = [m.start() for m in re.finditer(r"^\s+buffer_load_dwordx4 ", text, re.M)]
        assert len(loads) > 100
        for at in loads:                                       # a loop over the lanes: the load under a mask of its own
            assert "s_and_saveexec" not in "\n".join(text[:at].splitlines()[-3:])
