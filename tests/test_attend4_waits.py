"""Loads straight into LDS are counted by the kernels themselves, not by the compiler: whether all of them have been waited for where
their place is used for something else is read from the built code.  No GPU needed."""
import os
import re
import struct
import subprocess

import pytest

import paper_2511_13732_amd as pcg
from paper_2511_13732_amd import build as hip_build
from test_kernel_resources import ELF, EM_AMDGPU

OBJDUMP = os.path.join(os.path.dirname(os.path.realpath(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"))), "..", "llvm", "bin", "llvm-objdump")
OBJDUMP = OBJDUMP if os.path.exists(OBJDUMP) else "/opt/rocm/llvm/bin/llvm-objdump"
NOTHING = 64                                   # the counter has six bits


def code_of(path, part, folder):
    """{kernel: [(address, instruction, operands, address of a branch's end)]} of the kernels named `part` in the library at `path`."""
    blob, found = open(path, "rb").read(), {}
    at = blob.find(ELF, 1)
    while at >= 0:
        machine, = struct.unpack_from("<H", blob, at + 18)
        sections, = struct.unpack_from("<Q", blob, at + 40)
        each, count = struct.unpack_from("<HH", blob, at + 58)
        end = at + sections + each * count
        if machine == EM_AMDGPU and part.encode() in blob[at:end]:
            one = folder / "code"
            one.write_bytes(blob[at:end])
            text = subprocess.run([OBJDUMP, "-d", str(one)], capture_output=True, text=True, check=True).stdout
            code = []
            for line in text.splitlines():
                if head := re.match(r"([0-9a-f]+) <(\S+)>:$", line):
                    code, start = [], int(head[1], 16)
                    if f"{len(part)}{part}" in head[2]:
                        found[head[2]] = code
                elif step := re.match(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):(.*)$", line):
                    to = re.search(r"<[^>+]*(?:\+0x([0-9a-f]+))?>", step[4]) if step[1].startswith(("s_branch", "s_cbranch")) else None
                    code.append((int(step[3], 16), step[1], step[2], start + int(to[1] or "0", 16) if to else None))
        at = blob.find(ELF, at + 4)
    return found


def in_flight(code):
    """For every instruction how many vector-memory operations may be younger than the youngest load into LDS that may not be in yet on some
    way there, NOTHING if there is none, None where nobody comes."""
    place = {step[0]: i for i, step in enumerate(code)}
    state = [None] * len(code)
    state[0], todo = NOTHING, [0]
    while todo:
        i = todo.pop()
        _, name, operands, to = code[i]
        after = state[i]
        if name == "s_waitcnt":
            left = re.search(r"vmcnt\((\d+)\)", operands)
            if left and after >= int(left[1]):          # operations come in in their order
                after = NOTHING
        elif "load_lds" in name:
            after = 0
        elif name.startswith(("global_", "buffer_", "flat_", "scratch_")) and after < NOTHING:
            after = min(after + 1, NOTHING - 1)
        ends = [place[to]] if to is not None else []
        if name not in ("s_branch", "s_endpgm"):
            assert name not in ("s_setpc_b64", "s_swappc_b64")
            ends.append(i + 1)
        for j in ends:
            if state[j] is None or after < state[j]:
                state[j] = after
                todo.append(j)
    return state


def test_the_reading_of_code():
    """A loop of two loads that its end waits for, and one ahead of it that a way around the loop does not."""
    def code(*steps):
        return [(4 * i, *s.split(" ", 1), None) if i not in to else (4 * i, *s.split(" ", 1), 4 * to[i]) for i, s in enumerate(steps)]
    to = {1: 5, 4: 2}
    around = code("global_load_lds_dword x", "s_cbranch_scc1 5", "global_load_dword x", "s_waitcnt vmcnt(1)", "s_cbranch_scc0 2", "s_barrier x",
                  "s_endpgm x")
    assert in_flight(around) == [NOTHING, 0, 0, 1, NOTHING, 0, 0]
    to = {4: 2}
    through = code("global_load_lds_dword x", "s_nop 0", "global_load_dword x", "s_waitcnt vmcnt(1)", "s_cbranch_scc0 2", "s_barrier x", "s_endpgm x")
    assert in_flight(through) == [NOTHING, 0, 0, 1, NOTHING, NOTHING, NOTHING]


@pytest.mark.skipif(hip_build.sanitize_requested(), reason="the sanitizer build compiles for another optimisation level")
@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump beside hipcc")
def test_nothing_is_on_its_way_into_lds_but_a_piece_s_first_stage(tmp_path):
    """Waves of attend4_kernel meet with loads under way in one place, where the queries are handed over beside a piece's first stage.  Where the
    streams are joined, where the next piece begins and where the kernel ends, on every way there, nothing may be under way."""
    kernels = code_of(pcg.lib_path(), "attend4_kernel", tmp_path)
    assert len(kernels) == 20
    for name, code in kernels.items():
        state = in_flight(code)
        assert any("load_lds" in step[1] for step in code), name
        meets = [state[i] for i, step in enumerate(code) if step[1] == "s_barrier"]
        assert len([x for x in meets if x != NOTHING]) <= 1, (name, meets)
        assert all(state[i] in (NOTHING, None) for i, step in enumerate(code) if step[1] == "s_endpgm"), name
