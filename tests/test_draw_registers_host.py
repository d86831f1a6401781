"""The kernels that draw classes keep what they work on in registers: none is to spill a vector register (one kernel for all of a long row's forms,
bounded so that it did, gave wrong rows for a reason that its source does not show).  Read from what the compiler says of them; no GPU."""
import os
import re
import subprocess

from paper_1102_0183_amd import build


def test_kernels_that_draw_classes_spill_no_vector_register(tmp_path):
    out = os.path.join(str(tmp_path), "draws.s")
    src = [s for s in build.sources() if s.endswith("cnn355_draws.hip")][0]
    subprocess.run([build.HIPCC] + [f for f in build.FLAGS if f != "-fPIC"] + build.SOURCE_FLAGS.get(os.path.basename(src), []) +
                   ["--cuda-device-only", "-S", "-o", out, src], check=True, capture_output=True)
    text = open(out).read()
    kernels = re.findall(r"^\s*\.name:\s+(\S*k_draw\S*)$", text, flags=re.M)
    spills = re.findall(r"^\s*\.vgpr_spill_count:\s+(\d+)$", text, flags=re.M)
    scratch = re.findall(r"^\s*\.private_segment_fixed_size:\s+(\d+)$", text, flags=re.M)
    assert len(kernels) >= 27 and len(spills) == len(scratch) == len(kernels)
    assert [k for k, n, s in zip(kernels, spills, scratch) if int(n) or int(s)] == []
