"""Loads and stores that a source takes past the caches are so in the machine code.  (Two stores of the same value, one of
them so, behind a flag become one ordinary store: the flag then chooses nothing.)"""
import os
import re
import subprocess

import pytest

from paper_2606_18954_amd import build_lib

pytestmark = pytest.mark.skipif(not os.path.exists(build_lib.HIPCC), reason="hipcc not available")


def sources():
    for name in build_lib.SOURCES:
        with open(os.path.join(build_lib.CSRC, name), encoding="utf-8") as f:
            text = f.read()
        kinds = sorted(set(re.findall(r"__builtin_nontemporal_(load|store)", text)))
        if kinds:
            yield name, kinds


@pytest.mark.parametrize("name,kinds", list(sources()))
def test_what_goes_past_the_caches(name, kinds, tmp_path):
    out = tmp_path / "k.s"
    flags = [f for f in build_lib.CFLAGS if f != "-fPIC"]
    subprocess.run([build_lib.HIPCC, *flags, "-x", "hip", "-S", "--cuda-device-only", os.path.join(build_lib.CSRC, name), "-o",
                    str(out)], check=True, capture_output=True)
    text = out.read_text()
    for kind in kinds:
        assert re.search(rf"(global|flat|buffer)_{kind}_\S+ .* nt\b", text), (name, kind)
