"""The epilogue of the gated feed-forward block's 16-bit product kernels hands sums from lane to lane of a wave through LDS.
A wave's LDS accesses are carried out in the order they are issued in, so what makes that right is the order of the
compiled code: a half's sums are all written before the first of them is read, and all read before the next half's are
written.  Needs hipcc, no GPU."""
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_11490_amd", "csrc")


def _out_of_order(body):
    """Places behind the matrix instructions where a run of LDS writes is not one half's, whole."""
    tile = int(re.search(r"ELi(128|256)ELi\1E", body.split("\n", 1)[0]).group(1))
    half = (tile // 32 // 2) * (tile // 32)  # 16-byte pieces of a lane
    runs, last = [], ""
    for line in body[body.rindex("v_mfma"):].split("\n"):
        op = line.split(";")[0].strip()[:7]
        if op == "ds_writ":
            if last == "ds_writ":
                runs[-1] += 1
            else:
                runs.append(1)
        if op in ("ds_writ", "ds_read"):
            last = op
    assert runs and sum(runs) == 4 * half, (tile, runs)  # two halves, for tiles inside C and for the others
    return [r for r in runs if r != half]


@pytest.mark.parametrize("source", ["ffn_bf16.hip", "ffn_f16.hip"])
def test_halves_of_the_sums_follow_each_other(tmp_path, source):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc here")
    from paper_2502_11490_amd import build

    out = tmp_path / "kernel.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc] + flags + ["-S", "--cuda-device-only", os.path.join(CSRC, source), "-o", str(out)], check=True,
                   capture_output=True)
    bodies = re.findall(r"^(_Z\w*ffn_mfma16_kernel\w*:[^\n]*\n.*?)^\.Lfunc_end\d+:", out.read_text(), re.S | re.M)
    assert len(bodies) == 10, "five products in two tile sizes"
    bad = {b.split(":", 1)[0]: _out_of_order(b) for b in bodies}
    assert not {k: v for k, v in bad.items() if v}
