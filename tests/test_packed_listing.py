"""What the compiler makes of the packed cache's attention and of sampling, on the CPU: no inline assembly reads
a matrix result too early, no kernel calls a function, none keeps what its main loop uses in memory."""

import os
import re
import subprocess

import pytest

from paper_2608_00531_amd import build as pbuild
from test_matrix_waits import early_reads, kernels


@pytest.mark.skipif(not os.path.exists(pbuild.hipcc()), reason="hipcc not available")
@pytest.mark.parametrize("source", ["packed_attn.hip", "sample.hip", "kv_pack.hip"])
def test_listing(tmp_path, source):
    out = str(tmp_path / "listing.s")
    flags = [f for f in pbuild.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([pbuild.hipcc()] + flags + ["--cuda-device-only", "-S", "-I", pbuild.INCLUDE, "-I", pbuild.CSRC,
                                               os.path.join(pbuild.CSRC, source), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    found = kernels(text)
    assert found and not re.search(r"s_swappc|uses_dynamic_stack:\s+true|v_pk_(add|mul|fma)_f32", text)
    matrix = [name for name, blocks in found.items() if any(op.startswith("v_mfma") for _, code in blocks for _, op, _, _ in code)]
    assert bool(matrix) == (source == "packed_attn.hip")
    early = {name: lines for name, blocks in found.items() if (lines := early_reads(blocks))}
    assert not early, early
    # Registers in memory: the attention of few fp32 rows keeps one there, and none else but sampling does.
    spills = dict(re.findall(r"\.symbol:\s+(\w+)\.kd\n(?:.*\n)*?\s+\.vgpr_spill_count: (\d+)", text))
    assert spills and all(int(n) <= (2 if "few" in name else 0) for name, n in spills.items()) or source == "sample.hip", spills
