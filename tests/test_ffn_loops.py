"""The 16-bit product kernels of the gated feed-forward block write their matrix instructions as assembly statements, whose
wait states the compiler does not know.  What makes that right is checked in the compiled code of every kernel: in the
loop, the operands of a matrix instruction are written by LDS reads, or by a vector instruction at least 4 instructions
ahead (it needs 2 wait states), the accumulation registers by the matrix instructions only, nothing is spilled, and the
loop ends with the wait states of its last sums.  Needs hipcc, no GPU."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_11490_amd", "csrc")


def _registers(text):
    """The registers an operand names: 'v[2:5]' -> {('v', 2), ..., ('v', 5)}."""
    m = re.fullmatch(r"([va])(?:(\d+)|\[(\d+):(\d+)\])", text.strip())
    if not m:
        return set()
    lo, hi = (int(m.group(2)),) * 2 if m.group(2) else (int(m.group(3)), int(m.group(4)))
    return {(m.group(1), i) for i in range(lo, hi + 1)}


@pytest.mark.parametrize("source", ["ffn_bf16.hip", "ffn_f16.hip"])
def test_matrix_instructions_of_the_loops(tmp_path, source):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc here")
    from paper_2502_11490_amd import build

    out = tmp_path / "kernel.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", os.path.join(CSRC, source), "-o", str(out)], check=True,
                   capture_output=True)
    bodies = re.findall(r"^(_Z\w*ffn_mfma16_kernel\w*):[^\n]*\n(.*?)^\.Lfunc_end\d+:", out.read_text(), re.S | re.M)
    assert len(bodies) == 10, "five products in two tile sizes"
    for name, body in bodies:
        blocks, label = {}, ""
        for line in body.split("\n"):
            code = line.split(";")[0].strip()
            m = re.match(r"(\.LBB\w+):", code)
            if m:
                label = m.group(1)
            elif code and not code.startswith("."):
                blocks.setdefault(label, []).append(code)
        loops = [b for b in blocks.values() if any(c.startswith("v_mfma") for c in b)]
        assert len(loops) == 1, (name, "the matrix instructions are one block")
        loop = loops[0]
        assert sum(c.startswith("v_mfma") for c in loop) in (32, 128)
        assert not [c for c in loop if "scratch_" in c or "accvgpr" in c], name
        assert not any(c.startswith("v_mfma") for c in loop[:4]), (name, "the sums are set up ahead of the loop")
        writer = {}
        for i, code in enumerate(loop * 2):  # the second time round what the first left in the registers is known
            op, _, rest = code.partition(" ")
            operands = re.split(r",\s*(?![^\[]*\])", rest)
            if op.startswith("v_mfma"):
                for r in _registers(operands[1]) | _registers(operands[2]):
                    by, at = writer.get(r, ("ds_read", 0))
                    assert by.startswith("ds_read") or i - at >= 4, (name, code, by, i - at)
            if operands and not op.startswith(("s_", "buffer_", "ds_write", "global_store")):
                for r in _registers(operands[0]):
                    writer[r] = op, i
                    assert r[0] == "v" or op.startswith("v_mfma"), (name, code)
        last = max(i for i, c in enumerate(loop) if c.startswith("v_mfma"))
        assert any(c.startswith("s_nop 15") for c in loop[last + 1:]), (name, "wait states behind the last sums")
