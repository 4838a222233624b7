"""The build's own checks."""
from paper_1910_10892_amd import build

KERNEL = """mrfmp_attention.hip:36:1: remark: Function Name: %s [-Rpass-analysis=kernel-resource-usage]
mrfmp_attention.hip:36:1: remark:     TotalSGPRs: 58 [-Rpass-analysis=kernel-resource-usage]
mrfmp_attention.hip:36:1: remark:     VGPRs: 256 [-Rpass-analysis=kernel-resource-usage]
mrfmp_attention.hip:36:1: remark:     AGPRs: %d [-Rpass-analysis=kernel-resource-usage]
mrfmp_attention.hip:36:1: remark:     ScratchSize [bytes/lane]: %d [-Rpass-analysis=kernel-resource-usage]
mrfmp_attention.hip:36:1: remark:     Dynamic Stack: False [-Rpass-analysis=kernel-resource-usage]
mrfmp_attention.hip:36:1: remark:     Occupancy [waves/SIMD]: 1 [-Rpass-analysis=kernel-resource-usage]
"""


def test_kernels_with_scratch_memory_beside_accumulation_registers_are_found():
    report = "".join(KERNEL % k for k in (("plain", 0, 0), ("scratch", 0, 60), ("both", 16, 60), ("accumulation", 212, 0), ("last", 1, 4)))
    assert build.kernels_with_scratch_and_accumulation(report) == ["both", "last"]
    assert build.kernels_with_scratch_and_accumulation("") == []


def test_the_units_that_multiply_matrices_are_reported():
    assert set(build.UNIT_FLAGS) == {"mrfmp_attention.hip", "mrfmp_attention_bwd.hip"} and set(build.UNIT_FLAGS) <= set(build.LEARN_SOURCES)
