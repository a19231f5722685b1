"""What the sources of the sequence operators owe the compiler."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2210_08804_amd", "csrc")


def test_assembly_that_writes_m0_gives_it_back():
    """The compiler keeps m0 for itself: a statement that writes it without a word takes whatever it holds there."""
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*")):
        with open(path) as f:
            for statement in re.findall(r"\basm\b[^;]*;", f.read()):
                if "s_mov_b32 m0" in statement:
                    found += 1
                    kept = re.search(r"s_mov_b32 (%\d), m0", statement)
                    assert kept and statement.index(kept[0]) < statement.index("s_mov_b32 m0"), statement
                    assert re.findall(r"s_mov_b32 m0, (%\d)", statement)[-1] == kept[1], statement
    assert found
