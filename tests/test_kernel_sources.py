"""Rules of the instruction set that a kernel's results do not show, looked for in its source (no GPU)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_16007_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_a_group_of_warps_changes_its_registers_in_one_place():
    """setmaxnreg is for all four warps of a group together: one instance each way, behind a condition that holds for whole
    groups, and shares that add up to what the block was launched with."""
    text = source("toploc_attention_tc.cu")
    lower, raised = (list(re.finditer(w + r"_registers<(\w+)>\(\);", text)) for w in ("lower", "raise"))
    assert len(lower) == 1 and len(raised) == 1
    assert re.search(r"if \(warp < 8\) \{\s*$", text[:raised[0].start()])
    assert re.search(r"\} else \{\s*$", text[:lower[0].start()])
    value = {k: int(v) for k, v in re.findall(r"(k\w+Registers) = (\d+)", text)}
    assert 2 * value[raised[0][1]] + value[lower[0][1]] <= 3 * (65536 // 384 // 8 * 8)
