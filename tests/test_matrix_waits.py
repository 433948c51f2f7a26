"""No inline assembly reads a matrix instruction's result too early, on the CPU.

The compiler delays an instruction that reads a matrix instruction's result until it is there, but
not inline assembly, which it cannot see into. So on every path from a matrix instruction to
assembly that reads its result some other instruction must have read that result before. The
attention sources are compiled to assembly text with the build's flags, and every path of every kernel
is followed.
"""

import os
import re
import subprocess

import pytest

from paper_2608_00531_amd import build as pbuild


def registers(operand):
    m = re.match(r"([va])(?:\[(\d+):(\d+)\]|(\d+))$", operand)
    if not m:
        return []
    first, last = (m[2], m[3]) if m[2] else (m[4], m[4])
    return [m[1] + str(i) for i in range(int(first), int(last) + 1)]


def kernels(text):
    """name -> basic blocks: [label, [(line, opcode, operands, in inline assembly)]]"""
    found, blocks, asm = {}, None, False
    for number, line in enumerate(text.splitlines(), 1):
        if re.match(r"_Z\w+:", line):
            blocks = found.setdefault(line.split(":")[0], [[None, []]])
        elif line.startswith(".Lfunc_end"):
            blocks = None
        if blocks is None:
            continue
        s = line.strip()
        if s.startswith((";;#ASMSTART", ";;#ASMEND")):
            asm = s.startswith(";;#ASMSTART")
            continue
        label = re.match(r"(\.LBB\w+):", line)
        if label:
            blocks.append([label[1], []])
            continue
        s = s.split(";")[0].strip()
        if not s or s.startswith(".") or s.endswith(":"):
            continue
        op, _, rest = s.partition(" ")
        blocks[-1][1].append((number, op, [a.strip().split(" ")[0] for a in rest.split(",")], asm))
        if op.startswith(("s_branch", "s_cbranch", "s_endpgm")):
            blocks.append([None, []])
    return found


def early_reads(blocks):
    """Lines of assembly that may be the first to read a matrix result. State: register -> the matrix
    instructions (lines) whose result it may hold that nothing has read."""
    at = {label: i for i, (label, _) in enumerate(blocks) if label}
    bad = set()

    def walk(code, state):
        state = dict(state)
        for number, op, args, asm in code:
            vector = op.startswith("v_") and not op.startswith("v_mfma")
            read = [r for a in (args[1:] if op.startswith("v_") else args) for r in registers(a)]
            if vector and asm:
                bad.update(number for r in read if r in state)
            elif not op.startswith("v_mfma") and not asm:
                done = set().union(*(state.get(r, ()) for r in read)) if read else set()
                if done:
                    state = {r: left for r, ids in state.items() if (left := ids - done)}
            if op.startswith("v_mfma"):
                for r in registers(args[0]):
                    state[r] = frozenset([number])
            elif vector:
                for r in registers(args[0]):
                    state.pop(r, None)
        return state

    entry, todo = {0: {}}, [0]
    while todo:
        i = todo.pop()
        out = walk(blocks[i][1], entry[i])
        number, op, args, _ = blocks[i][1][-1] if blocks[i][1] else (0, "", [], False)
        following = [at[args[0]]] if op.startswith(("s_branch", "s_cbranch")) else []
        if not op.startswith(("s_branch", "s_endpgm")) and i + 1 < len(blocks):
            following.append(i + 1)
        for j in following:
            new = dict(entry.get(j, {}))
            for r, ids in out.items():
                new[r] = new.get(r, frozenset()) | ids
            if j not in entry or new != entry[j]:
                entry[j] = new
                todo.append(j)
    return sorted(bad)


LISTING = """
_Zkernel:
	v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]
	s_cbranch_vccz .LBB0_2
	{visible}
.LBB0_2:
	;;#ASMSTART
	v_max3_f32 v30, v30, v{reg}, v{reg}
	;;#ASMEND
	s_endpgm
.Lfunc_end0:
"""


def test_the_check_itself():
    """A result that one of two paths leaves unread; one read on both; another register's."""
    def lines(listing):
        return [early_reads(b) for b in kernels(listing).values()]
    both = LISTING.replace("\ts_cbranch_vccz .LBB0_2\n", "")
    assert lines(LISTING.format(visible="v_max_f32_e32 v31, v3, v3", reg=5)) == [[8]]
    assert lines(both.format(visible="v_max_f32_e32 v31, v3, v3", reg=5)) == [[]]
    assert lines(both.format(visible="v_max_f32_e32 v31, v16, v16", reg=5)) == [[7]]
    assert lines(LISTING.format(visible="s_nop 0", reg=16)) == [[]]


@pytest.mark.skipif(not os.path.exists(pbuild.hipcc()), reason="hipcc not available")
@pytest.mark.parametrize("source", ["tree_attn.hip", "prompt_attn.hip"])
def test_assembly_never_reads_a_matrix_result_first(tmp_path, source):
    out = str(tmp_path / "listing.s")
    flags = [f for f in pbuild.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([pbuild.hipcc()] + flags + ["--cuda-device-only", "-S", "-I", pbuild.INCLUDE, "-I", pbuild.CSRC,
                                               os.path.join(pbuild.CSRC, source), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        found = kernels(f.read())
    assert any(op.startswith("v_mfma") for blocks in found.values() for _, code in blocks for _, op, _, _ in code)
    early = {name: lines for name, blocks in found.items() if (lines := early_reads(blocks))}
    assert not early, early
