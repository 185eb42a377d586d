"""The build's reading of hipcc's report on registers, CPU-only."""
from paper_2206_08888_amd import build

REPORT = """
k.hip:9:1: remark: Function Name: _Z3onev [-Rpass-analysis=kernel-resource-usage]
k.hip:9:1: remark:     VGPRs: 12 [-Rpass-analysis=kernel-resource-usage]
k.hip:9:1: remark:     SGPRs Spill: 3 [-Rpass-analysis=kernel-resource-usage]
k.hip:9:1: remark:     VGPRs Spill: 0 [-Rpass-analysis=kernel-resource-usage]
k.hip:30:1: remark: Function Name: _Z3twov [-Rpass-analysis=kernel-resource-usage]
k.hip:30:1: remark:     SGPRs Spill: 0 [-Rpass-analysis=kernel-resource-usage]
k.hip:30:1: remark:     VGPRs Spill: 17 [-Rpass-analysis=kernel-resource-usage]
"""


def test_vector_spills():
    assert build.vector_spills(REPORT) == [("_Z3onev", 0), ("_Z3twov", 17)]
    assert build.vector_spills("") == []
