"""What the operators' compiled kernels hold of a CU, read from the metadata of the library built here: nothing spilled, and as many
workgroups to a CU as the launches count on.
"""
import struct
import subprocess

import pytest

from paper_2410_20650_amd import build
from test_kernel_resources import LDS_OF_A_CU, REGISTERS_OF_A_SIMD_LANE, kernel_metadata

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects():
    """One of each translation unit."""
    with open(build.BUILT_LIB, "rb") as f:
        data = f.read()
    at = data.find(MAGIC)
    while at >= 0:
        (entries,) = struct.unpack_from("<Q", data, at + 24)
        place = at + 32
        for _ in range(entries):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            if b"gfx950" in data[place + 24:place + 24 + length]:
                yield data[at + offset:at + offset + size]
            place += 24 + length
        at = data.find(MAGIC, at + len(MAGIC))


@pytest.fixture(scope="module")
def kernels():
    found = [k for elf in code_objects() for k in kernel_metadata(elf)]
    names = subprocess.run(["c++filt"], input="\n".join(k[".name"] for k in found), capture_output=True, text=True,
                           check=True).stdout.split("\n")
    return dict(zip((n.replace("void ", "").replace("nz::", "") for n in names), found))


def of(kernels, begin):
    chosen = {n: k for n, k in kernels.items() if n.startswith(begin)}
    assert chosen, begin
    return chosen


@pytest.mark.parametrize("begin", ["embedding_", "gated_", "linear_adapters_", "adapter_"])
def test_nothing_is_spilled(kernels, begin):
    for name, k in of(kernels, begin).items():
        assert k[".vgpr_spill_count"] == 0 and k[".sgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


def registers(k):
    """Of a lane, in eights; the ones for sums come from the same 512."""
    return (k[".vgpr_count"] + 7) // 8 * 8


# (the linear layer's two workgroups of eight waves; two of the gated block's tiles of 128, one of its tiles of 256)
@pytest.mark.parametrize("begin, workgroups", [("linear_adapters_", 2), ("gated_gradients_", 2), ("gated_kernel", 1),
                                               *((f"gated_kernel<(GatedForm){form}, 128, 2>", 2) for form in range(3))])
def test_workgroups_of_a_cu(kernels, begin, workgroups):
    for name, k in of(kernels, begin).items():
        waves = k[".max_flat_workgroup_size"] // 64
        assert workgroups * k[".group_segment_fixed_size"] <= LDS_OF_A_CU, name
        assert registers(k) * workgroups * waves // 4 <= REGISTERS_OF_A_SIMD_LANE, name
