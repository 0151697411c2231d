"""As many workgroups of attend4_kernel find room on a compute unit as its grid has for each: what is launched for two or four and finds room
for one or three works in uneven waves.  From the metadata beside the built code.  No GPU needed."""
import re

import pytest

pytest.importorskip("msgpack")

import paper_2511_13732_amd as pcg
from paper_2511_13732_amd import build as hip_build
from test_kernel_resources import kernels

# by the rows' type, elements of a head (at most) and blocks of 16 rows
GROUPS = {("t", 64, 1): 4, ("t", 64, 2): 3, ("t", 64, 3): 2, ("t", 128, 1): 2, ("t", 128, 2): 2, ("t", 128, 3): 2,
          ("f", 64, 1): 4, ("f", 64, 2): 3, ("f", 128, 1): 3, ("f", 128, 2): 2}


@pytest.mark.skipif(hip_build.sanitize_requested(), reason="the sanitizer build compiles for another optimisation level")
def test_a_compute_unit_has_room_for_the_workgroups_that_are_launched_for_it():
    found = {}
    for k in kernels(pcg.lib_path()):
        if name := re.search(r"14attend4_kernelI([tf])Li(\d+)ELi(\d+)ELi(\d)E", k[".name"]):
            found[name[1], int(name[2]), int(name[3]), int(name[4])] = k
    assert sorted(found) == sorted((*of, pages) for of in GROUPS for pages in (1, 2))
    for of, k in found.items():
        groups = GROUPS[of[:3]]
        assert k[".max_flat_workgroup_size"] == 256                    # a wave on each of the four SIMDs
        assert groups * k[".group_segment_fixed_size"] <= 160 * 1024, (of, k[".group_segment_fixed_size"])
        assert groups * ((k[".vgpr_count"] + 7) // 8 * 8) <= 512, (of, k[".vgpr_count"])
