"""What the compiler made of the tiled products of operands in 8 bits (no GPU needed)."""
import re

import pytest

from tests.test_built_code import _registers, kernels  # noqa: F401


def bodies(kernels, name):
    found = [b for n, b in kernels.items() if re.search(name, n)]
    assert len(found) == 1
    return [line.split("//")[0].strip() for line in found[0].splitlines() if re.match(r"\s+[a-z]+_", line)]


TILES = [(r"product_kernelIaLb1ELb1ELi%dELi%dE.*Lb1E%sE" % (t, t, kind), "v_mfma_i32_16x16x64_i8") for kind in ("DF16b", "DF16_", "f") for t in (256, 128, 64)]


# (and the tile of gradients in 32 bits where larger ones would leave most compute units without one)
@pytest.mark.parametrize("name,product", TILES + [(r"product_pair_kernelIfLi32ELi64E", "v_mfma_f32_16x16x4_f32")])
def test_written_products_are_left_where_they_are_and_wait_for_their_operands(kernels, name, product):  # noqa: F811
    # as for the operands of 16 bits: behind a matrix instruction, up to a branch or the waits that follow the last one, no
    # accumulator is read elsewhere or spilled; two instructions lie between the vector instruction that writes an operand and its use
    behind, seen, written = False, 0, []
    for line in bodies(kernels, name):
        op, _, operands = line.partition(" ")
        if op == product:
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
