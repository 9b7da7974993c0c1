"""What the compiler made of the kernels, read from the code objects of the built library (no GPU needed)."""
import os
import re
import subprocess

import pytest

LLVM = "/opt/rocm/llvm/bin"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Disassembly of every kernel of the library, by its mangled name."""
    from paper_2506_11277_amd import build
    objdump = os.path.join(LLVM, "llvm-objdump")
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(build.LIB):
        build.build_lib()
    folder = tmp_path_factory.mktemp("code")
    lib = folder / "lib.so"
    lib.write_bytes(open(build.LIB, "rb").read())
    subprocess.run([objdump, "--offloading", str(lib)], cwd=folder, check=True, stdout=subprocess.DEVNULL)
    found = {}
    for name in os.listdir(folder):
        if "gfx950" not in name:
            continue
        text = subprocess.run([objdump, "-d", "--no-show-raw-insn", str(folder / name)], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"^[0-9a-f]+ (?=<.*>:$)", text, flags=re.M)[1:]:
            label, _, body = part.partition(">:\n")
            found[label[1:]] = body
    return found


@pytest.mark.parametrize("kernel", ["gemm_fused16_kernelILi%dELi0E" % s for s in range(2, 10)] + ["gemm_fused_kernelILi%dE" % s for s in (1, 10, 16, 20)] +
                         ["gemm_halves_kernelILi4E", "gemm_halves16_kernelILi7E", "gemm_eighths_kernelILi7E", "gemm_eighths_whole_kernelI"] +
                         ["gemm_eighths_passes_kernelI", "gemm_passes_kernelI"])
def test_c_has_streaming_and_plain_stores(kernels, kernel):
    # columns of C on 64-byte boundaries are stored past the caches, others through them: both kinds of store have to be in
    # the code of every kernel that writes C from its accumulators (identical but for that, they are easily made one)
    bodies = [b for name, b in kernels.items() if kernel in name]
    stores = [re.findall(r"global_store_dwordx2 .*", b) for b in bodies]
    stores = [s for s in stores if s]                       # (split-k and dump variants write no C)
    assert stores, sorted(kernels)[:5]
    for s in stores:
        assert any(" nt" in line for line in s) and any(" nt" not in line for line in s), (kernel, s[:4])


@pytest.mark.parametrize("tile", [256, 128, 64])
@pytest.mark.parametrize("kind", ["DF16b", "DF16_", "f"])
def test_written_products_are_left_where_they_are(kernels, kind, tile):
    # The tiled products' matrix instructions are written out, so the compiler does not know that their results take a while: behind
    # one, up to a branch or the waits that follow the last one, it must not read an accumulator register elsewhere or spill one.
    name = r"product_(kernelI%sLb[01]ELb[01]ELi%dELi%dE.*Lb1E|pair_kernelI%sLi%dE)" % (kind, tile, tile, kind, tile)
    bodies = [b for n, b in kernels.items() if re.search(name, n)]
    assert len(bodies) >= (0 if kind == "f" and tile == 256 else 3)
    for body in bodies:
        lines = [line.strip() for line in body.splitlines() if re.match(r"\s+[a-z]+_", line)]
        behind, seen = False, 0
        for line in lines:
            if line.startswith("v_mfma"):
                behind, seen = True, seen + 1
            elif line.startswith(("s_branch", "s_cbranch", "s_endpgm")) or line.split("//")[0].split() == ["s_nop", "15"]:
                behind = False
            elif behind:
                assert not line.startswith(("v_accvgpr_read", "v_accvgpr_mov", "scratch_store")), line
        assert seen


def _registers(operands):
    out = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", operands):
        out |= {kind + str(i) for i in range(int(a), int(b) + 1)}
    return out | {kind + a for kind, a in re.findall(r"\b([va])(\d+)\b", operands)}


@pytest.mark.parametrize("tile", [256, 128, 64])
@pytest.mark.parametrize("kind", ["DF16b", "DF16_", "f"])
def test_written_products_wait_for_their_operands(kernels, kind, tile):
    # ... nor does it know that a matrix instruction wants two wait states behind the vector instruction that writes an operand
    name = r"product_(kernelI%sLb[01]ELb[01]ELi%dELi%dE.*Lb1E|pair_kernelI%sLi%dE)" % (kind, tile, tile, kind, tile)
    for body in [b for n, b in kernels.items() if re.search(name, n)]:
        written = []                                    # registers written by the last two instructions, if by vector ones
        for line in body.splitlines():
            if not re.match(r"\s+[a-z]+_", line):
                continue
            op, _, operands = line.split("//")[0].strip().partition(" ")
            if op.startswith("v_mfma"):
                assert not any(w & _registers(operands) for w in written), line
            vector = op.startswith("v_") and not op.startswith("v_mfma")
            written = written[-1:] + [_registers(operands.split(",")[0]) if vector else set()]
            if op == "s_nop" and int(operands.strip(), 0) >= 1:
                written = []
