"""The build-time guard of test_isa_staged_copies.py for the kernels that read a quantized cache."""
import os
import subprocess

import pytest

from paper_2409_16997_amd import build as hip_build
from test_isa_staged_copies import faults, instructions


@pytest.mark.timeout(600)
@pytest.mark.parametrize("source", [s for s in hip_build.SOURCES if s.startswith("intfa_cache_")])
def test_every_staged_copy_has_its_wait_states(source, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = tmp_path / "kernels.s"
    subprocess.run([hipcc, *flags, "-S", "--cuda-device-only", "-I", hip_build.INCLUDE, "-I", hip_build.CSRC, os.path.join(hip_build.CSRC, source), "-o", str(out)],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    copies, bad = faults(list(instructions(out.read_text().splitlines())))
    assert copies > 0
    assert not bad, f"{len(bad)} of {copies} copies, the first: {bad[0]}"
