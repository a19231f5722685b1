"""The kernels over 4-bit pages as they are compiled."""
import re

import pytest

from test_seq_kernels import kernels  # noqa: F401

BESIDE = {(1, 1): 4, (2, 1): 4, (3, 1): 3, (4, 1): 3, (8, 1): 2, (1, 2): 4, (2, 2): 3, (3, 2): 2, (4, 2): 2}          # waves of a SIMD, which have 512 registers in all


@pytest.mark.parametrize("groups,tiles", sorted(BESIDE))
@pytest.mark.parametrize("dtype", ["DF16_", "DF16b"])
def test_few_rows_stay_in_their_registers(kernels, dtype, groups, tiles):  # noqa: F811
    """A register that does not fit is read back with a wait for all loads under way, and those of the next step are to stay under way."""
    mine = [v for k, v in kernels.items() if f"packed_few_kernelI{dtype}Li{groups}ELi{tiles}E" in k]
    assert len(mine) == 1
    vgprs, spilled = mine[0]
    assert spilled == 0 and vgprs <= 512 // BESIDE[groups, tiles] // 8 * 8


@pytest.mark.parametrize("groups", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", ["DF16_", "DF16b"])
def test_many_rows_of_up_to_128_values_stay_in_their_registers(kernels, dtype, groups):  # noqa: F811
    mine = [v for k, v in kernels.items() if re.search(rf"packed_kernelI{dtype}Li{groups}ELi\dE", k)]
    assert len(mine) == 2
    for vgprs, spilled in mine:
        assert vgprs <= 256 and spilled <= (1 if groups == 4 else 0)


def test_norms_and_appends_need_no_scratch_memory(kernels):  # noqa: F811
    mine = {k: v for k, v in kernels.items() if re.search("norm_kernel|norm_grad_kernel|norm_join_kernel|append_kernel|read_kernel", k)}
    assert len(mine) >= 30 and all(spilled == 0 for _, spilled in mine.values()), mine
