"""Properties of the machine code of the kernels between two attention calls: nothing spilled, no packed float32, and the
logit rules' registers within the eight waves per SIMD that hide their counting."""
import os
import re
import subprocess

import pytest

from paper_2606_18954_amd import build_lib

pytestmark = pytest.mark.skipif(not os.path.exists(build_lib.HIPCC), reason="hipcc not available")


@pytest.mark.parametrize("name,kernels,most", [("slots.hip", 4, 128), ("qkv.hip", 12, 128), ("logits.hip", 3, 64)])
def test_kernels_do_not_spill(name, kernels, most, tmp_path):
    out = tmp_path / "k.s"
    flags = [f for f in build_lib.CFLAGS if f != "-fPIC"]
    src = os.path.join(build_lib.CSRC, name)
    subprocess.run([build_lib.HIPCC, *flags, "-x", "hip", "-S", "--cuda-device-only", src, "-o", str(out)], check=True,
                   capture_output=True)
    text = out.read_text()
    scratch = [int(x) for x in re.findall(r"ScratchSize:\s+(\d+)", text)]
    registers = [int(x) for x in re.findall(r"; NumVgprs:\s+(\d+)", text)]
    assert len(scratch) == kernels and not any(scratch), scratch
    assert max(registers) <= most, registers
    assert not re.search(r"v_pk_(add|mul|fma)_f32", text)
