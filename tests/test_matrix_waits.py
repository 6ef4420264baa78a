"""Every use of a bf16 matrix product in the kernels built here comes late enough: the compiler
has left out wait states where a branch stands between."""
import os

import pytest

from paper_2606_23743_amd import build

from . import matrix_waits

pytestmark = [pytest.mark.cpu, pytest.mark.skipif(matrix_waits.objdump() is None, reason="needs llvm-objdump")]

PRODUCT = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]"


def listing(*lines):
    """Instructions of four bytes each from address 0x1000 on; a branch names its target's number."""
    out = ["0000000000001000 <kernel>:"]
    for i, line in enumerate(lines):
        op, _, rest = line.partition(" ")
        target = f" <kernel+0x{4 * int(rest):x}>" if op.startswith(("s_cbranch", "s_branch")) else ""
        out.append(f"\t{line}    // {0x1000 + 4 * i:012X}: 00000000{target}")
    return "\n".join(out)


@pytest.mark.parametrize("late,lines", [
    (2, [PRODUCT, "s_cmp_eq_u32 s0, s1", "s_cbranch_scc1 5", "v_mov_b32 v20, 0", "s_endpgm", "v_mul_f32 v4, v3, v5", "s_endpgm"]),
    (3, [PRODUCT, "s_cmp_eq_u32 s0, s1", "s_cbranch_scc1 5", "v_mov_b32 v20, 0", "v_add_f32 v4, v0, v0", "s_nop 7", "s_endpgm"]),
    (0, [PRODUCT, "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], v[4:7]", "s_endpgm"]),
    (6, [PRODUCT, "s_nop 5", "global_store_dwordx4 v[20:21], v[0:3], off", "s_endpgm"]),
    (None, [PRODUCT, "s_nop 7", "v_mul_f32 v4, v3, v5", "s_endpgm"]),
    (None, [PRODUCT, PRODUCT, "s_nop 7", "v_mul_f32 v4, v3, v5", "s_endpgm"]),
    (None, [PRODUCT, "s_cmp_eq_u32 s0, s1", "s_cbranch_scc1 4", "s_endpgm", "s_nop 5", "v_mul_f32 v4, v3, v5", "s_endpgm"]),
    (None, [PRODUCT, "v_mov_b32 v4, v5", "s_branch 0"]),
])
def test_the_scan_finds_early_uses(late, lines):
    (name, body), = matrix_waits.kernels(listing(*lines))
    found = matrix_waits.early_uses(body)
    assert name == "kernel" and [w for _, _, w in found] == ([] if late is None else [late])


def test_no_kernel_uses_a_product_early(tmp_path):
    if not os.path.exists(build.LIB):
        pytest.skip("the library is not built")
    seen, early = 0, []
    for code in matrix_waits.code_objects(build.LIB):
        for name, body in matrix_waits.kernels(matrix_waits.disassemble(code, str(tmp_path))):
            seen += any(matrix_waits.PRODUCT.match(op) for _, op, _, _ in body)
            early += [(name, hex(a), hex(b), w) for a, b, w in matrix_waits.early_uses(body)]
    assert seen > 100 and not early, early[:8]
