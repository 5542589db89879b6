"""The loads to LDS of the experts' large tiles set m0 in inline assembly, which cannot say so to
the compiler: nothing else in these kernels may use it.  Checked in the assembly that the build's
flags give (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_1503_08294_amd import build

# instructions that read m0 without naming it
READS = re.compile(r"\b(s_movrel|v_movrel|s_sendmsg|ds_gws|ds_\w*addtid|v_interp|"
                   r"buffer_load\w*.*\blds\b|s_ttrace|ds_ordered)")


@pytest.mark.parametrize("source", ["experts_bf16.hip", "experts_f16.hip"])
def test_m0_is_only_set_for_the_loads(source, tmp_path):
    out = str(tmp_path / "kernels.s")
    subprocess.run([build.hipcc(), *build.FLAGS, "-S", "--cuda-device-only",
                    os.path.join(build.CSRC, source), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        lines = [line.split(";")[0].strip() for line in f]
    lines = [line for line in lines if line and not line.startswith(".")]
    loads = 0
    for i, line in enumerate(lines):
        assert not READS.search(line), line
        if re.search(r"\bm0\b", line):
            assert re.fullmatch(r"s_mov_b32 m0, s\d+", line), line
            assert lines[i + 1] == "s_nop 0", lines[i:i + 3]
            assert lines[i + 2].startswith("global_load_lds_dword"), lines[i:i + 3]
            loads += 1
    assert loads == sum(line.startswith("global_load_lds_dword") for line in lines) > 0
