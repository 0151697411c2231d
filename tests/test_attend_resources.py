"""The kernels around a step's forward pass are in the built library, without scratch memory and in the registers and shared
memory that their launch bounds ask for, from the metadata beside their code.  No GPU needed."""
import pytest

pytest.importorskip("msgpack")

import paper_2511_13732_amd as pcg
from paper_2511_13732_amd import build as hip_build
from test_kernel_resources import kernels


@pytest.mark.skipif(hip_build.sanitize_requested(), reason="the sanitizer build compiles for another optimisation level")
@pytest.mark.parametrize("part,variants", [("pages_step_kernel", 2), ("pages_step_large_kernel", 1), ("pages_slots_kernel", 1),
                                           ("cache_write_kernel", 1), ("attend_thin_kernel", 4), ("attend_thick_kernel", 20),
                                           ("attend_prompt_kernel", 8), ("attend_join_kernel", 10)])
def test_kernels_fit(part, variants):
    mine = [k for k in kernels(pcg.lib_path()) if f"{len(part)}{part}" in k[".name"]]
    assert len(mine) == variants
    for k in mine:
        assert not k[".vgpr_spill_count"] and not k[".private_segment_fixed_size"], k[".name"]
        # two workgroups a compute unit, but for those whose keys and values fill its shared memory: 512 registers a lane on each of
        # four SIMDs
        if "attend" in part and k[".group_segment_fixed_size"] <= 80 * 1024:
            waves = -(-2 * k[".max_flat_workgroup_size"] // 64 // 4)
            assert k[".vgpr_count"] * waves <= 512, k[".name"]
