"""What the kernels' sources keep to where a fault could not be shown by running it (no GPU needed)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2608_23658_b200", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


SPLIT = [n for n in sorted(os.listdir(CSRC)) if n.endswith((".cu", ".cuh")) and 'asm volatile("setmaxnreg' in source(n)]


@pytest.mark.parametrize("name", SPLIT)
def test_a_register_split_is_one_instruction_for_all_warps_of_a_warpgroup(name):
    """setmaxnreg is .aligned: the four warps of a warpgroup execute the same instruction, so it hangs on no condition of a single warp."""
    text = source(name)
    for m in re.finditer(r'asm volatile\("setmaxnreg', text):
        line = text[text.rfind("\n", 0, m.start()) + 1:m.start()].strip()
        assert not line, f"{name}: a condition stands in front of setmaxnreg: {line}"
        before = text[:m.start()].rstrip().rsplit("\n", 1)[-1].strip()
        assert not re.search(r"warp\s*[!=]=\s*\d", before) and not before.endswith("set_up();"), f"{name}: setmaxnreg for one warp: {before}"


def test_the_rows_kernel_gives_every_copy_a_chance_to_land_when_it_gives_up():
    """A bulk copy that is still under way when its CTA has left lands in the shared memory of the next one."""
    text = source("ekv_rows.cuh")
    kernel = text[text.index("rows_kernel("):]
    teardown = kernel[kernel.rindex("if (*sh.abort_flag()) {"):kernel.rindex("tcgen05_dealloc")]
    for bar in ("K_FULL", "V_RAW", "Q_FULL"):                       # what its tma_load_3d complete on
        assert re.search(r"mbar_wait\([^;]*\b" + bar + r"\b", teardown), bar
