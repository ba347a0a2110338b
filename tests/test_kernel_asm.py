"""What inline assembly in the kernels writes, it names: the compiler keeps values of its own elsewhere then."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2201_00194_amd", "csrc")


def test_assembly_that_writes_m0_names_it():
    found = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        for statement in re.findall(r"\basm\b[^;]*?\(.*?\);", open(path).read(), re.S):
            if re.search(r"s_mov_b32 m0\b", statement):
                found += 1
                assert '"m0"' in statement.rsplit(":", 1)[1], (os.path.basename(path), statement)
    assert found >= 2
