"""What the source of the chunk kernels has to keep and no run would show."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_18121_b200", "csrc")


def test_a_warpgroup_changes_its_registers_by_one_instruction():
    """All warps of a group have to meet the same setmaxnreg: one place for each group, under a condition that its warps share."""
    text = open(os.path.join(CSRC, "ec_chunk_attention.cu")).read()
    assert len(re.findall(r"setmaxnreg\.dec", text)) == 1 and len(re.findall(r"setmaxnreg\.inc", text)) == 1
    assert re.search(r"if \(warp < 4\) \{\n\s*asm volatile\(\"setmaxnreg\.dec\.sync\.aligned\.u32 (\d+);\"\);", text)
    few, many = (int(re.search(r"setmaxnreg\." + k + r"\.sync\.aligned\.u32 (\d+)", text).group(1)) for k in ("dec", "inc"))
    assert 4 * few + 8 * many <= 12 * 168                      # more than the launch was given would wait for good
