"""What the compiler made of the tiled products of operands in 8 bits (no GPU needed)."""
import re

import pytest

from tests.test_built_code import _registers, kernels  # noqa: F401


def bodies(kernels, kind, tile):
    found = [b for n, b in kernels.items() if re.search(r"product_kernelIaLb1ELb1ELi%dELi%dE.*Lb1E%sE" % (tile, tile, kind), n)]
    assert len(found) == 1
    return [line.split("//")[0].strip() for line in found[0].splitlines() if re.match(r"\s+[a-z]+_", line)]


@pytest.mark.parametrize("tile", [256, 128, 64])
@pytest.mark.parametrize("kind", ["DF16b", "DF16_", "f"])
def test_written_products_are_left_where_they_are_and_wait_for_their_operands(kernels, kind, tile):  # noqa: F811
    # as for the operands of 16 bits: behind a matrix instruction, up to a branch or the waits that follow the last one, no
    # accumulator is read elsewhere or spilled; two instructions lie between the vector instruction that writes an operand and its use
    behind, seen, written = False, 0, []
    for line in bodies(kernels, kind, tile):
        op, _, operands = line.partition(" ")
        if op == "v_mfma_i32_16x16x64_i8":
            behind, seen = True, seen + 1
            assert not any(w & _registers(operands) for w in written), line
        elif line.startswith(("s_branch", "s_cbranch", "s_endpgm")) or line.split() == ["s_nop", "15"]:
            behind = False
        elif behind:
            assert not line.startswith(("v_accvgpr_read", "v_accvgpr_mov", "scratch_store")), line
        vector = op.startswith("v_") and not op.startswith("v_mfma")
        written = written[-1:] + [_registers(operands.split(",")[0]) if vector else set()]
        if op == "s_nop" and int(operands.strip(), 0) >= 1:
            written = []
    assert seen
