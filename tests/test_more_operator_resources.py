"""What the compiled kernels of the norm, the cache, its attention and the logits hold of a CU: nothing spilled, and as many waves as their comments count on."""
import pytest

from test_kernel_resources import LDS_OF_A_CU, REGISTERS_OF_A_SIMD_LANE
from test_operator_resources import kernels, of, registers  # noqa: F401 (a fixture)


@pytest.mark.parametrize("begin", ["norm_", "append_", "attend_", "logits_"])
def test_nothing_is_spilled(kernels, begin):  # noqa: F811
    for name, k in of(kernels, begin).items():
        assert k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


# waves to a SIMD
@pytest.mark.parametrize("begin, waves", [("attend_few_kernel<64u", 4), ("attend_few_kernel<128u", 3), ("attend_some_kernel<64u", 3), ("attend_some_kernel<128u", 2),
                                          ("attend_many_kernel<64u", 3), ("attend_many_kernel<128u", 2), ("norm_back_kernel", 4), ("logits_kernel", 8)])
def test_waves_of_a_simd(kernels, begin, waves):  # noqa: F811
    for name, k in of(kernels, begin).items():
        of_workgroup = (k[".max_flat_workgroup_size"] + 255) // 256     # waves to a SIMD
        assert registers(k) * waves <= REGISTERS_OF_A_SIMD_LANE, name
        assert waves // of_workgroup * k[".group_segment_fixed_size"] <= LDS_OF_A_CU, name
