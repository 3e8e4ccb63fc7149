"""A matrix product's result may be read only some cycles after the product was issued.  The compiler keeps that distance for the
instructions that it chooses, not for the text of inline assembly: the attention kernels over the 4-bit cache, which take their
maxima straight from matrix products, hold no vector instruction there."""
import os
import re
import subprocess

import pytest

from paper_2512_24449_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.parametrize("source", ["fp4_attention.hip", "fp4_tiles.hip"])
def test_no_vector_instruction_in_inline_assembly(source, tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path / "kernels.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC, *flags, "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "--offload-device-only", "-S",
                    "-o", str(out), os.path.join(build.CSRC, source)], check=True, capture_output=True)
    text = out.read_text()
    assert len(re.findall(r"^\s+v_mfma", text, re.M)) > 32, "the kernels' matrix products were not found"
    inline = "\n".join(re.findall(r"#ASMSTART(.*?)#ASMEND", text, re.S))
    assert not re.findall(r"^\s*v_.*", inline, re.M)
