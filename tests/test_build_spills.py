"""The build looks at what ptxas reports of the microscaled products: a kernel of theirs that spills is named, others may."""
from paper_1602_02830_b200 import build

LINE = "ptxas warning : Registers are spilled to local memory in function '%s', %d bytes spill stores, %d bytes spill loads"


def test_spilling_kernels_are_named():
    pair, few, norm = "_ZN50_GLOBAL__N__4ba268b09k_mx_pairILi0ELi1ELi256EEEvNS_8PairArgsE", "_ZN1_8k_mx_fewILi0ELb1EEEvNS_7FewArgsE", "_ZN1_12k_block_normI6__halfLi4EEEvNS_8NormArgsE"
    assert build.spilled("") == [] and build.spilled(LINE % (norm, 44, 60)) == []
    log = "\n".join(["some warning", LINE % (pair, 12, 16), LINE % (norm, 44, 60), LINE % (few, 8, 8)])
    assert build.spilled(log) == [f"{pair}: 12 bytes stored, 16 loaded", f"{few}: 8 bytes stored, 8 loaded"]


def test_the_flag_that_reports_them_is_given():
    assert "-Xptxas=-warn-spills" in build.NVCC_FLAGS
