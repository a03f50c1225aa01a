"""The products with an epilogue, the gradient through an activation and the 8-bit checkpoints, on the host: what
they refuse, what they launch (read from the fake HIP runtime)."""
import pytest

from tests.act_tiles import TILES
from tests.fake_hip import ADDR, calls
from tests.libqe import need_lib


def product_launches(qe, hip, products):
    got = []
    for gated, m, n, k in products:
        hip.clear()
        ld = (k + 15) // 16 * 16
        if gated:
            st = qe.qe_fp8_gemm_gated(ADDR, 0, ld, ADDR, ADDR, 0, ld, m, n, k, ADDR, ADDR, ADDR, qe.ACT_SILU, ADDR, qe.BF16,
                                      n, stream=0)
        else:
            st = qe.qe_fp8_gemm_act(ADDR, 0, ld, ADDR, 0, ld, m, n, k, ADDR, ADDR, None, ADDR, qe.BF16, n, stream=0)
        assert st == "OK", st
        got.append([w[2] for w in hip.log("launch")])
    return got


def test_products_get_their_kernel():
    got = calls(product_launches, [list(t[1:]) for t in TILES])
    for t, names in zip(TILES, got):
        assert len(names) == 1 and t[0] in names[0], (t, names)


# gated, m, n, k: up to 16 rows, or few blocks of 16 x 16 outputs and a long reduction; and what is just past that
ROWS = [(False, 1, 4096, 14336), (True, 16, 14336, 4096), (False, 17, 256, 1025), (True, 256, 256, 1025), (False, 512, 256, 12289)]
TILED = [(False, 17, 256, 1024), (True, 257, 256, 1025), (False, 257, 256, 12288), (False, 513, 256, 12289), (True, 512, 256, 12289)]


def test_few_blocks_split_the_reduction():
    assert all("act_rows_kernel" in n for n, in calls(product_launches, [list(c) for c in ROWS]))
    assert all("act_rows_kernel" not in n for n, in calls(product_launches, [list(c) for c in TILED]))


OK = dict(a=16, fmt_a=0, lda=32, b=16, fmt_b=0, ldb=32, m=4, n=40, k=20, sa=16, sb=16, c=16, c_dtype=1, ldc=40)


def act(qe, epi="default", **kw):
    v = {**OK, **kw}
    e = qe.make_epilogue() if epi == "default" else epi
    return qe.qe_fp8_gemm_act(v["a"], v["fmt_a"], v["lda"], v["b"], v["fmt_b"], v["ldb"], v["m"], v["n"], v["k"], v["sa"],
                              v["sb"], e, v["c"], v["c_dtype"], v["ldc"], stream=0)


def gated(qe, gate=None, up=None, b2=16, s2=16, which=0, **kw):
    v = {**OK, **kw}
    return qe.qe_fp8_gemm_gated(v["a"], v["fmt_a"], v["lda"], v["b"], b2, v["fmt_b"], v["ldb"], v["m"], v["n"], v["k"],
                                v["sa"], v["sb"], s2, which, v["c"], v["c_dtype"], v["ldc"], gate, up, stream=0)


BAD_OPERANDS = [dict(a=0), dict(b=0), dict(c=0), dict(sa=0), dict(sb=0), dict(fmt_a=2), dict(fmt_b=-1), dict(c_dtype=2),
                dict(m=-1), dict(n=-1), dict(k=-1), dict(ldc=39), dict(lda=16), dict(lda=40), dict(ldb=16), dict(ldb=33),
                dict(lda=1 << 23), dict(ldb=1 << 23), dict(a=8), dict(b=24), dict(c=17), dict(c=18, c_dtype=0),
                dict(m=1 << 31), dict(n=1 << 31, ldc=1 << 31), dict(k=1 << 24, lda=1 << 24, ldb=1 << 24),
                dict(m=1 << 25, n=1 << 20, ldc=1 << 20)]


@pytest.mark.parametrize("bad", BAD_OPERANDS, ids=str)
def test_products_refuse_bad_operands(bad):
    qe = need_lib()
    assert act(qe, **bad) == "INVALID_ARG"
    assert gated(qe, **bad) == "INVALID_ARG"


def test_gated_refuses():
    qe = need_lib()
    i8 = qe.make_saved(qe.SAVED_I8, 16, 40, 16, 2)
    for bad in (dict(b2=0), dict(b2=8), dict(s2=0), dict(which=5), dict(which=-1), dict(gate=i8), dict(up=i8),
                dict(gate=i8, up=qe.make_saved(qe.SAVED_BF16, 16, 40)),
                dict(gate=qe.make_saved(qe.SAVED_I8, 16, 39, 16, 2), up=i8),
                dict(gate=i8, up=qe.make_saved(qe.SAVED_I8, 16, 40, 16, 1)),
                dict(gate=qe.make_saved(3, 16, 40, 16, 2), up=qe.make_saved(3, 16, 40, 16, 2))):
        assert gated(qe, **bad) == "INVALID_ARG", bad


def test_epilogue_refuses():
    qe = need_lib()
    e = qe.make_epilogue
    for bad in (e(act=5), e(act=-1), e(bias=16, bias_dtype=2), e(bias=17, bias_dtype=qe.BF16), e(bias=18, bias_dtype=qe.F32),
                e(residual=16, residual_dtype=qe.BF16, ld_residual=39), e(residual=18, residual_dtype=qe.F32, ld_residual=40),
                e(residual=16, residual_dtype=3, ld_residual=40), e(saved=qe.make_saved(qe.SAVED_BF16, 17, 40)),
                e(saved=qe.make_saved(qe.SAVED_BF16, 0, 40)), e(saved=qe.make_saved(qe.SAVED_BF16, 16, 39)),
                e(saved=qe.make_saved(qe.SAVED_I8, 16, 40, 0, 2)), e(saved=qe.make_saved(qe.SAVED_I8, 16, 40, 16, 1)),
                e(saved=qe.make_saved(7, 16, 40, 16, 2))):
        assert act(qe, epi=bad) == "INVALID_ARG"


def test_empty_products_do_nothing():
    qe = need_lib()
    for empty in (dict(m=0), dict(n=0)):
        assert act(qe, a=0, b=0, c=0, **empty) == "OK" and act(qe, epi=None, **empty) == "OK"
        assert gated(qe, a=0, b=0, c=0, **empty) == "OK"


def grad(qe, **kw):
    v = dict(dd=16, dt=1, ld=40, rows=4, cols=40, act=4, z=qe.make_saved(qe.SAVED_I8, 16, 40, 16, 2), u=None,
             meta=qe.FP8Meta(16, 16, 16, 4, 0, 0, 0, 16), q_row=16, ld_row=80, q_col=16, ld_col=4, snap=16, dz=16, dzt=0,
             ld_dz=80, dbias=None, mode=0, ws=None)
    v.update(kw)
    return qe.qe_act_grad(v["dd"], v["dt"], v["ld"], v["rows"], v["cols"], v["act"], v["z"], v["u"], v["meta"], v["q_row"],
                          v["ld_row"], v["q_col"], v["ld_col"], v["snap"], v["dz"], v["dzt"], v["ld_dz"], v["dbias"],
                          v["mode"], v["ws"], stream=0)


def test_grad_refuses():
    qe = need_lib()
    s, i8 = qe.make_saved, qe.make_saved(qe.SAVED_I8, 16, 40, 16, 2)
    for bad in (dict(dd=0), dict(dd=17), dict(dd=18, dt=0), dict(dt=2), dict(ld=39), dict(rows=-1), dict(cols=-1), dict(act=5),
                dict(z=None), dict(z=s(0)), dict(z=s(qe.SAVED_I8, 16, 39, 16, 2)), dict(z=s(qe.SAVED_I8, 16, 40, 16, 1)),
                dict(z=s(qe.SAVED_BF16, 17, 40)), dict(u=s(qe.SAVED_BF16, 16, 40)), dict(u=s(qe.SAVED_I8, 0, 40, 16, 2)),
                dict(meta=qe.FP8Meta(16, 16, 16, 0, 0, 0, 0, 16)), dict(meta=qe.FP8Meta(16, 0, 16, 4, 0, 0, 0, 16)),
                dict(meta=None), dict(meta=None, q_row=None, q_col=None), dict(ld_row=39), dict(u=i8, ld_row=79), dict(ld_col=3),
                dict(dz=18), dict(dzt=3), dict(ld_dz=39), dict(u=i8, ld_dz=79), dict(dbias=16), dict(dbias=16, ws=18),
                dict(dbias=18, ws=16), dict(dbias=16, ws=16, mode=2), dict(u=i8, dbias=16, ws=16),
                dict(rows=1 << 31, ld_col=1 << 31), dict(rows=1 << 25, cols=1 << 25, ld=1 << 25, ld_row=1 << 25, ld_col=1 << 25,
                                                         ld_dz=1 << 25, z=s(qe.SAVED_BF16, 16, 1 << 25))):
        assert grad(qe, **bad) == "INVALID_ARG", bad


def test_checkpoint_refuses():
    qe = need_lib()
    good = dict(x=16, dt=0, ld=40, rows=4, cols=40, s=qe.make_saved(qe.SAVED_I8, 16, 40, 16, 2))
    for bad in (dict(x=0), dict(x=18), dict(dt=2), dict(ld=39), dict(rows=-1), dict(cols=-1), dict(s=None),
                dict(s=qe.make_saved(qe.SAVED_BF16, 16, 40)), dict(s=qe.make_saved(qe.SAVED_I8, 0, 40, 16, 2)),
                dict(s=qe.make_saved(qe.SAVED_I8, 16, 40, 0, 2)), dict(s=qe.make_saved(qe.SAVED_I8, 16, 39, 16, 2)),
                dict(s=qe.make_saved(qe.SAVED_I8, 16, 40, 16, 1)), dict(rows=1 << 31)):
        v = {**good, **bad}
        assert qe.qe_act_save(v["x"], v["dt"], v["ld"], v["rows"], v["cols"], v["s"], stream=0) == "INVALID_ARG", bad
        assert qe.qe_act_restore(v["s"], v["rows"], v["cols"], v["x"], v["dt"], v["ld"], stream=0) == "INVALID_ARG", bad


def grad_launches(qe, hip, cases):
    got = []
    for rows, cols, two, bias, snap in cases:
        hip.clear()
        z = qe.make_saved(qe.SAVED_I8, ADDR, cols, ADDR, (cols + 31) // 32)
        meta = qe.FP8Meta(ADDR, ADDR, ADDR, 4, 0, 1, 0, ADDR)
        st = qe.qe_act_grad(ADDR, qe.BF16, cols, rows, cols, qe.ACT_SILU, z, z if two else None, meta, ADDR, 2 * cols, ADDR, rows,
                            ADDR if snap else None, dbias=ADDR if bias else None, workspace=ADDR if bias else None, stream=0)
        assert st == "OK", st
        got.append([w[2].split("kernel")[0].split("115")[-1].split("116")[-1] for w in hip.log("launch")])
    return got


def test_grad_launches():
    """One kernel, one more for the bias gradient; an empty gradient writes its snapshot and its (zero) bias gradient."""
    got = calls(grad_launches, [[100, 100, False, False, True], [100, 100, True, False, True], [100, 100, False, True, True],
                                [0, 100, False, True, True], [0, 100, False, False, False], [100, 0, False, True, False]])
    assert got == [["act_grad_"], ["act_grad_"], ["act_grad_", "bias_grad_"], ["act_grad_", "bias_grad_"], [], []]


def test_struct_sizes():
    """The binding's structs have the sizes the C compiler gives the header's."""
    import ctypes
    import os
    import shutil
    import subprocess
    import tempfile
    from tests.libqe import ROOT
    qe = need_lib()
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src = '#include <stdio.h>\n#include "qe.h"\nint main(void) { printf("%zu %zu\\n", sizeof(qe_saved), sizeof(qe_epilogue)); return 0; }\n'
    with tempfile.TemporaryDirectory() as td:
        c, exe = os.path.join(td, "s.c"), os.path.join(td, "s")
        open(c, "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe], check=True)
        got = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in got] == [ctypes.sizeof(qe.Saved), ctypes.sizeof(qe.Epilogue)]


# name part, workgroups a compute unit is to hold (of a SIMD's 512 registers, given in eights, and 160 KB of LDS)
OCCUPANCY = [("act_grad_kernelILb1ELb1ELi2ELi128ELi256E", 3), ("act_grad_kernelILb0ELb1ELi2ELi64ELi512E", 3),
             ("act_ring_kernelILb1ELi0ELi0ELi64ELi64ELi4E", 2), ("act_ring_kernelILb0ELi0ELi0ELi128ELi128ELi2E", 2),
             ("act_rows_kernelILb1ELi0ELi0ELi1ELi8E", 2), ("act_large_kernelILb1ELi0ELi0ELi256ELi256E", 1)]


@pytest.mark.parametrize("part,workgroups", OCCUPANCY, ids=lambda v: str(v))
def test_workgroups_per_compute_unit(part, workgroups):
    from tests.kernel_resources import kernels
    k, = [k for n, k in kernels(need_lib().LIB_PATH).items() if part in n]
    waves = k[".max_flat_workgroup_size"] // 256  # on each SIMD
    assert 512 // ((k[".vgpr_count"] + 7) // 8 * 8) >= workgroups * max(1, waves)
    assert k[".group_segment_fixed_size"] * workgroups <= 160 * 1024
