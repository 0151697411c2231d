"""What the attention kernels' instructions written by hand tell the compiler.  No GPU needed."""
import os
import re

import paper_2511_13732_amd as pcg

CSRC = os.path.join(os.path.dirname(pcg.__file__), "csrc")


def test_no_instruction_written_by_hand_changes_m0_unseen():
    """m0 is a register that the compiler moves values to for its own use; one that is reserved cannot be named as changed, so a statement
    that needs it takes it as an operand."""
    found = 0
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for asm in re.findall(r"asm volatile\((.*?)\);", text, re.S):
            code = asm.split("::")[0]
            assert not re.search(r"\bm0\b", code), (name, asm)
            if "global_load_lds" in code:
                assert '"{m0}"' in asm, (name, asm)
                found += 1
    assert found >= 4


def test_loads_written_by_hand_wait_for_scalars_that_the_vector_unit_wrote():
    """Five wait states between a vector instruction that writes a scalar register and a load that takes its address from it: the
    compiler keeps them for its own loads only."""
    found = 0
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for asm in re.findall(r"asm volatile\((.*?)\);", text, re.S):
            if "global_load_lds" in asm:
                assert asm.lstrip().startswith('"s_nop 4\\n'), (name, asm)
                found += 1
    assert found >= 4
