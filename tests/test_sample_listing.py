"""What the compiler makes of sampling, on the CPU. Its kernels keep registers in memory (the search for places,
and a bf16 row's general way), but no loop that counts a row's entries into a histogram does, nor the loops that read
bf16 rows in vectors of 16 bytes."""

import os
import re
import subprocess

import pytest

from paper_2608_00531_amd import build as pbuild


@pytest.mark.skipif(not os.path.exists(pbuild.hipcc()), reason="hipcc not available")
def test_loops_over_a_row_keep_nothing_in_memory(tmp_path):
    out = str(tmp_path / "listing.s")
    flags = [f for f in pbuild.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([pbuild.hipcc()] + flags + ["--cuda-device-only", "-S", "-I", pbuild.INCLUDE, "-I", pbuild.CSRC,
                                               os.path.join(pbuild.CSRC, "sample.hip"), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    found = re.findall(r"^(_ZN\S*sample_(?:f32|bf16)\S*):[^\n]*\n(.*?)^\.Lfunc_end", text, re.S | re.M)
    assert len(found) == 2
    for name, body in found:
        # Innermost loops by their header: a block's comment names it, the header's own its label.
        loops, counts = {}, set()
        for block in re.split(r"^(?=\.LBB|; %bb)", body, flags=re.M)[1:]:
            head = block.split("\n\n")[0]
            label = re.match(r"\.L(BB\w+):", block)
            inside = re.findall(r"Header=(BB\w+)", block.split("\n")[0]) or re.findall(r"Parent Loop (BB\w+)", head)
            if label and "Loop Header" in head:
                inside = [label.group(1)]
            if not inside:
                continue
            ops = re.findall(r"^\t([a-z]\w+)", block, re.M)
            loops.setdefault(inside[-1], []).extend(ops)
            if sum(op.startswith("ds_add") for op in ops) or sum(op == "global_load_dwordx4" for op in ops):
                counts.add(inside[-1])
        assert len(counts) >= 3, name
        for loop in counts:
            assert not any(op.startswith("scratch_") for op in loops[loop]), (name, loop)
