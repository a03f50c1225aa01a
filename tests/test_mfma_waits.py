"""The inline-assembly matrix instructions of the block-scaled products, in the built library: nothing the compiler put between
or behind them (a copied or spilled accumulator, say) touches a result that is not there yet."""
import os

import pytest

from tests import mfma_waits
from tests.libqe import need_lib

needs_objdump = pytest.mark.skipif(not os.path.exists(mfma_waits.OBJDUMP), reason="no disassembler")


def listing(*texts, branches={}):
    """Lines as the disassembler prints them, four bytes each; branches: {line: the line it goes to}."""
    tail = lambda i: " <k+0x%x>" % (4 * branches[i]) if i in branches else ""  # noqa: E731
    return mfma_waits.parse("0000000000001000 <k>:\n" + "".join("\t%s // %012X: BF800000%s\n" % (t, 0x1000 + 4 * i, tail(i))
                                                                  for i, t in enumerate(texts)))["k"]


MFMA = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[2:9], v[10:17], a[0:3], v18, v19 op_sel_hi:[0,0,0]"


def test_a_result_that_is_touched_too_early_is_found():
    """By reads and writes, behind too few wait states, through a branch and around a loop; not by the next product."""
    read = "v_accvgpr_read_b32 v1, a2"
    early = lambda *texts, **kw: mfma_waits.too_early(listing(*texts, **kw))  # noqa: E731
    assert early(MFMA, read) == [(read, 0)] and early(MFMA, "s_nop 10", read) == [(read, 11)]
    assert early(MFMA, "v_accvgpr_write_b32 a3, 0") and early(MFMA, "ds_write_b128 v1, a[0:3]")
    assert not early(MFMA, "s_nop 11", read) and not early(MFMA, "v_accvgpr_read_b32 v1, a4")
    assert not early(MFMA, MFMA, "s_nop 15", read)
    assert early(MFMA, "s_cbranch_scc0 1", "s_nop 15", read, branches={1: 3}) == [(read, 1)]
    assert early("s_nop 0", read, "s_nop 0", MFMA, "s_branch 0", branches={4: 0}) == [(read, 2)]
    assert early(MFMA, "s_getpc_b64 s[4:5]", "s_add_u32 s4, s4, 0x10", "s_addc_u32 s5, s5, 0", "s_setpc_b64 s[4:5]", "s_endpgm", read) == [(read, 4)]


@needs_objdump
def test_no_block_product_touches_a_sum_too_early():
    kernels = 0
    for elf in mfma_waits.code_objects(need_lib().LIB_PATH):
        if b"block_large_kernel" not in elf:
            continue
        for name, body in mfma_waits.listings(elf).items():
            if any("v_mfma" in text for _, text, _ in body):
                assert not mfma_waits.too_early(body), name
                kernels += 1
    assert kernels == 4 * 15  # pairs of formats; few rows, seven small tiles, two large ones in two types
