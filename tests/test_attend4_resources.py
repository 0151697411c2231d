"""The kernels of rows on their way into a cache and of attention over 4 bits are in the built library, without scratch memory and in the
registers that two workgroups a compute unit leave each.  No GPU needed."""
import pytest

pytest.importorskip("msgpack")

import paper_2511_13732_amd as pcg
from paper_2511_13732_amd import build as hip_build
from test_kernel_resources import kernels


@pytest.mark.skipif(hip_build.sanitize_requested(), reason="the sanitizer build compiles for another optimisation level")
@pytest.mark.parametrize("part", ["append_kernel", "append4_kernel", "cache4_read_kernel", "attend4_kernel", "attend4_join_kernel"])
def test_kernels_fit(part):
    mine = [k for k in kernels(pcg.lib_path()) if f"{len(part)}{part}" in k[".name"]]
    assert mine
    for k in mine:
        assert not k[".vgpr_spill_count"] and not k[".private_segment_fixed_size"], k[".name"]
        if part == "attend4_kernel":
            assert 2 * k[".group_segment_fixed_size"] <= 160 * 1024 and k[".vgpr_count"] <= 256, k[".name"]
