"""Wait states of the gfx950 machine code that no hardware interlock and no compiler check provides.

Direct-to-LDS copies are written as inline assembly: a scalar write of M0 (where in LDS the copy goes),
then the copy.  The copy needs one wait state behind that write; where the compiler emits the pair itself
it puts one there, but it does not look inside inline assembly.  The address of a copy in scalar registers
that a vector instruction wrote needs five.  Both are read from the disassembly of every source that copies.
"""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_18954_amd", "csrc")
HIPCC = "/opt/rocm/bin/hipcc"
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
COPY = "global_load_lds_dwordx4"

pytestmark = pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(OBJDUMP)),
                                reason="hipcc or llvm-objdump not available")


def _machine_code(name, tmp_path):
    """Instructions of the source's device code, as the library build compiles it."""
    from paper_2606_18954_amd import build_lib
    obj = tmp_path / (name + ".o")
    flags = [f for f in build_lib.CFLAGS if f != "-fPIC"]
    subprocess.run([HIPCC, *flags, "-x", "hip", "-c", "--cuda-device-only", "--no-gpu-bundle-output",
                    os.path.join(CSRC, name), "-o", str(obj)], check=True, capture_output=True)
    text = subprocess.run([OBJDUMP, "-d", str(obj)], check=True, capture_output=True, text=True).stdout
    return [re.sub(r"\s*//.*", "", x).strip() for x in text.splitlines() if x.startswith("\t")]


def _scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$", operand) or re.match(r"s(\d+)$", operand)
    return set(range(int(m[1]), int(m[m.lastindex]) + 1)) if m else set()


def _states(instruction):
    m = re.match(r"s_nop (\d+)$", instruction)
    return 1 + int(m[1]) if m else 1


@pytest.mark.parametrize("name", ["seg_attn.hip", "mq_attn.hip", "mq_fp4_attn.hip", "fp4_attn.hip", "equiv.hip"])
def test_copies_wait_for_m0_and_their_address(name, tmp_path):
    code = _machine_code(name, tmp_path)
    copies = 0
    for i, x in enumerate(code):
        if not x.startswith(COPY):
            continue
        copies += 1
        # (the write is part of the copy's statement, so nothing branches in between)
        gap = 0
        j = i - 1
        while not re.search(r"\bm0\b", code[j]):
            gap += _states(code[j])
            j -= 1
        assert re.match(r"s_mov_b32 m0, ", code[j]), (name, code[j:i + 1])
        assert gap >= 1, (name, code[j:i + 1])
        address = set().union(*(_scalars(o) for o in re.split(r"[ ,]+", x)[1:]))
        gap, j = 0, i - 1
        while gap < 5 and j >= 0 and address:
            op, _, rest = code[j].partition(" ")
            if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
                assert not address & _scalars(rest.split(",")[0].strip()), (name, code[j:i + 1])
            gap += _states(code[j])
            j -= 1
    assert copies, name


def test_no_other_source_copies_to_lds():
    """A new source with such copies has to join the list above."""
    listed = {"seg_attn.hip", "mq_attn.hpp", "fp4_attn.hip", "equiv.hip", "attn_dev.hpp"}
    users = {f for f in os.listdir(CSRC)
             if re.search(r"\bdma16(_cached|_at)?\(|" + COPY, open(os.path.join(CSRC, f)).read())}
    assert users == listed
