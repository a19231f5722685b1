"""The kernels of the sequence operators as they are written and as they are compiled."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2210_08804_amd import binding

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
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


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """By name of a kernel, (vector registers, those of them that did not fit)."""
    d = tmp_path_factory.mktemp("objects")
    lib = shutil.copy(binding.LIB_PATH, d)
    subprocess.run([os.path.join(LLVM, "llvm-objdump"), "--offloading", lib], check=True, capture_output=True)
    found = {}
    for f in sorted(os.listdir(d)):
        if "gfx950" in f:
            notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", os.path.join(d, f)], check=True, capture_output=True, text=True).stdout
            for kernel in notes.split(".agpr_count:")[1:]:
                of = lambda key: int(re.search(rf"\.{key}:\s*(\d+)", kernel)[1])  # noqa: B023, E731
                found[re.search(r"\.name:\s*(\S+)", kernel)[1]] = of("vgpr_count"), of("vgpr_spill_count")
    return found


@pytest.mark.parametrize("exact", [0, 1])
@pytest.mark.parametrize("tiles", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", ["DF16_", "DF16b"])
def test_attention_of_up_to_128_values_stays_in_its_registers(kernels, dtype, tiles, exact):
    """Two waves a SIMD have 256 each.  A register that does not fit is read back with a wait for all loads under way; at 128
    values one is."""
    mine = [v for k, v in kernels.items() if f"attend_kernelI{dtype}Li{tiles}ELb{exact}E" in k]
    assert len(mine) == 1
    vgprs, spilled = mine[0]
    assert vgprs <= 256 and spilled <= (1 if tiles == 4 else 0)
