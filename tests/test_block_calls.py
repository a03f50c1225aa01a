"""The block-scaled cast and products and the norms around a residual sum, on the host: what they refuse, what they launch."""
import pytest

from tests.fake_hip import ADDR, calls
from tests.libqe import need_lib


def blocked(qe, cols=40, **kw):
    v = dict(data=16, ld=cols, exps=16, ld_exps=(cols + 127) // 128, fmt=0, block_rows=1)
    v.update(kw)
    return qe.make_blocked(v["data"], v["ld"], v["exps"], v["ld_exps"], v["fmt"], v["block_rows"])


def matrix(qe, cols=40, **kw):
    v = dict(data=16, ld=cols, dtype=0)
    v.update(kw)
    return qe.make_matrix(v["data"], v["ld"], v["dtype"])


BAD_MATRIX = [dict(data=0), dict(data=18), dict(data=17, dtype=1), dict(ld=39), dict(dtype=2)]
BAD_BLOCKED = [dict(data=0), dict(exps=0), dict(ld=39), dict(ld_exps=0), dict(fmt=2), dict(fmt=-1), dict(block_rows=0), dict(block_rows=64)]


def test_cast_refuses():
    qe = need_lib()

    def cast(rows=4, cols=40, inp="", row="", col=""):
        return qe.qe_quantize_fp8_block(matrix(qe) if inp == "" else inp, rows, cols, blocked(qe) if row == "" else row,
                                        blocked(qe, 4) if col == "" else col, stream=0)
    for bad in BAD_MATRIX:
        assert cast(inp=matrix(qe, **bad)) == "INVALID_ARG", bad
    for bad in BAD_BLOCKED:
        assert cast(row=blocked(qe, **bad), col=None) == "INVALID_ARG", bad
        assert cast(col=blocked(qe, 4, **dict(bad, **({"ld": 3} if "ld" in bad else {}))), row=None) == "INVALID_ARG", bad
    for bad in (dict(inp=None), dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31), dict(col=blocked(qe, 4, fmt=1)),
                dict(col=blocked(qe, 4, block_rows=128)), dict(rows=1 << 30, cols=1 << 10, inp=matrix(qe, 1 << 10), row=blocked(qe, 1 << 10),
                                                               col=None)):
        assert cast(**bad) == "INVALID_ARG", bad
    assert cast(rows=0, inp=None) == "OK" and cast(cols=0, inp=None) == "OK"


OK = dict(m=4, n=40, k=200, c=16, c_dtype=1, ldc=40)


def product(qe, a="", b="", epi=None, **kw):
    v = {**OK, **kw}
    op = blocked(qe, 200, ld=208, ld_exps=4)
    return qe.qe_fp8_gemm_block(op if a == "" else a, op if b == "" else b, v["m"], v["n"], v["k"], epi, v["c"], v["c_dtype"], v["ldc"], stream=0)


def test_product_refuses():
    qe = need_lib()
    for bad in (dict(data=0), dict(data=8), dict(exps=0), dict(exps=18), dict(ld=192), dict(ld=216), dict(ld=1 << 23), dict(ld_exps=2),
                dict(ld_exps=6), dict(ld_exps=1 << 23), dict(fmt=2), dict(fmt=-1), dict(block_rows=2), dict(block_rows=0)):
        op = blocked(qe, 200, **{**dict(ld=208, ld_exps=4), **bad})
        assert product(qe, a=op) == "INVALID_ARG" and product(qe, b=op) == "INVALID_ARG", bad
    for bad in (dict(a=None), dict(b=None), dict(c=0), dict(c=17), dict(c=18, c_dtype=0), dict(c_dtype=2), dict(m=-1), dict(n=-1), dict(k=-1),
                dict(ldc=39), dict(k=209), dict(k=513), dict(m=1 << 31), dict(n=1 << 31, ldc=1 << 31), dict(m=1 << 25, n=1 << 10, ldc=1 << 10)):
        assert product(qe, **bad) == "INVALID_ARG", bad
    e = qe.make_epilogue
    for bad in (e(act=5), e(bias=18, bias_dtype=qe.F32), e(residual=16, residual_dtype=qe.BF16, ld_residual=39),
                e(saved=qe.make_saved(qe.SAVED_I8, 16, 40, 16, 1))):
        assert product(qe, epi=bad) == "INVALID_ARG"
    for empty in (dict(m=0), dict(n=0)):
        assert product(qe, a=None, b=None, c=0, **empty) == "OK"


def desc(qe, **kw):
    v = dict(post_norm=True, post_weight=16, pre_norm=True, pre_weight=16, gate=16, ld_gate=40, gate_rows=4)
    v.update(kw)
    return qe.make_residual(**v)


BAD_DESC = [dict(post_eps=0.0), dict(pre_eps=-1.0), dict(post_eps=float("nan")), dict(weight_dtype=2), dict(post_weight=18), dict(pre_weight=18),
            dict(gate=18), dict(gate_dtype=2), dict(ld_gate=39), dict(gate_rows=0), dict(post_norm=2), dict(pre_norm=-1)]


def test_norm_refuses():
    qe = need_lib()

    def norm(rows=4, cols=40, x="", y="", d="", r="", h="", row="", col="", post=16, pre=32):
        m = lambda v: matrix(qe) if v == "" else v  # noqa: E731
        return qe.qe_residual_norm(m(x), m(y), rows, cols, desc(qe) if d == "" else d, m(r),
                                   matrix(qe, data=32) if h == "" else h, blocked(qe) if row == "" else row, blocked(qe, 4) if col == "" else col, post, pre,
                                   stream=0)
    for bad in BAD_DESC:
        assert norm(d=desc(qe, **bad)) == "INVALID_ARG", bad
    for bad in BAD_MATRIX:
        for name in "xyrh":
            assert norm(**{name: matrix(qe, **bad)}) == "INVALID_ARG", (name, bad)
    for bad in BAD_BLOCKED + [dict(block_rows=128)]:
        assert norm(row=blocked(qe, **bad), col=None) == "INVALID_ARG", bad
    plain = desc(qe, post_norm=False, pre_norm=False)
    for bad in (dict(d=None), dict(x=None, y=None), dict(rows=-1), dict(cols=16385, x=matrix(qe, 16385)), dict(rows=1 << 31),
                dict(d=plain), dict(d=plain, h=None, row=None, col=None, post=None), dict(y=None, post=16), dict(d=desc(qe, post_norm=False)),
                dict(post=18), dict(pre=18), dict(post=32), dict(pre=None), dict(r=None), dict(y=None, post=None, r=None, d=desc(qe, x_scale=0.5)),
                dict(y=None, post=None, r=None, h=matrix(qe)), dict(h=matrix(qe)), dict(h=matrix(qe), col=None, row=None),
                dict(r=matrix(qe, data=48, ld=41), y=matrix(qe, data=48)), dict(r=matrix(qe, dtype=1)), dict(h=matrix(qe, data=48, dtype=1), y=matrix(qe, data=48)),
                dict(col=blocked(qe, 4, fmt=1)), dict(col=blocked(qe, 4, block_rows=128)),
                dict(col=blocked(qe, 4, ld=3))):
        assert norm(**bad) == "INVALID_ARG", bad  # (h over x or r, which the transposed codes are made from)
    assert norm(rows=0) == "OK" and norm(cols=0) == "OK"


def test_norm_grad_refuses():
    qe = need_lib()

    def grad(rows=4, cols=40, dr="", dh="", r="", y="", d="", post=16, pre=16, dx="", dy="", dpost=16, dpre=32, dgate=48, ld=40, mode=0, ws=16):
        m = lambda v, at: matrix(qe, data=at) if v == "" else v  # noqa: E731
        return qe.qe_residual_norm_grad(m(dr, 16), m(dh, 32), m(r, 48), m(y, 64), rows, cols, desc(qe) if d == "" else d, post, pre, m(dx, 80), m(dy, 96),
                                        dpost, dpre, dgate, mode, ws, ld, stream=0)
    for bad in BAD_DESC:
        assert grad(d=desc(qe, **bad)) == "INVALID_ARG", bad
    for bad in BAD_MATRIX:
        for name in ("dr", "dh", "r", "y", "dx", "dy"):
            assert grad(**{name: matrix(qe, **bad)}) == "INVALID_ARG", (name, bad)
    for bad in (dict(d=None), dict(dr=None, dh=None), dict(rows=-1), dict(cols=16385), dict(d=desc(qe, pre_norm=False)), dict(r=None), dict(pre=None),
                dict(post=None), dict(y=None), dict(y=None, dy=None), dict(mode=2), dict(dh=None), dict(d=desc(qe, pre_weight=None)),
                dict(d=desc(qe, post_weight=None)), dict(d=desc(qe, post_norm=False)), dict(d=desc(qe, gate=None)), dict(ld=39), dict(ws=None),
                dict(ws=18), dict(dpost=18), dict(dpre=18), dict(dgate=18), dict(post=18), dict(pre=18), dict(rows=1 << 27),
                dict(dx=matrix(qe, data=16, dtype=1)), dict(dx=matrix(qe, data=32, ld=41)), dict(dy=matrix(qe, data=16, ld=48)),
                dict(dx=matrix(qe, data=48)), dict(dx=matrix(qe, data=64)), dict(dy=matrix(qe, data=48)), dict(dy=matrix(qe, data=64)),
                dict(dx=matrix(qe, data=96)), dict(dpost=32), dict(dpost=48), dict(dgate=32)):
        assert grad(**bad) == "INVALID_ARG", bad


def launches(qe, hip, cases):
    got = []
    for kind, rows, cols, args in cases:
        hip.clear()
        m = qe.make_matrix(ADDR, max(cols, 1), qe.BF16)
        b = lambda c: qe.make_blocked(ADDR, c, ADDR, (c + 127) // 128, 0)  # noqa: E731
        d = qe.make_residual(post_norm=True, post_weight=ADDR, pre_norm=True, pre_weight=ADDR, gate=ADDR if args.get("gate") else None,
                             ld_gate=cols, gate_rows=args.get("gate", 0))
        if kind == "cast":
            st = qe.qe_quantize_fp8_block(m, rows, cols, b(cols) if args.get("row", True) else None, b(rows) if args.get("col") else None, stream=0)
        elif kind == "norm":
            st = qe.qe_residual_norm(m, m, rows, cols, d, m, None, b(cols), b(rows) if args.get("col") else None, ADDR, 2 * ADDR, stream=0)
        else:
            o, o2 = (qe.make_matrix(i * ADDR, max(cols, 1), qe.BF16) for i in (2, 3))
            st = qe.qe_residual_norm_grad(m, m, m, m, rows, cols, d, ADDR, ADDR, o, o2, ADDR if args.get("sums") else None,
                                          2 * ADDR if args.get("sums") else None, 3 * ADDR if args.get("gate") else None, qe.INIT, ADDR, stream=0)
        assert st == "OK", st
        got.append([w[2].split("kernel")[0].lstrip("_ZN2qe1GLOBAL").lstrip("_0123456789") for w in hip.log("launch")])
    return got


def test_launches():
    """A cast is one kernel, a norm one and one more for its transposed codes; a gradient one, one more for the sums of columns, one
    for the sums over the rows of gates where they are more than 256 or have more than 16 chunks, and one where few long rows leave
    the columns to it."""
    got = calls(launches, [["cast", 100, 300, {"col": 1}], ["cast", 100, 300, {"row": False}], ["norm", 100, 300, {}], ["norm", 100, 300, {"col": 1}],
                           ["grad", 100, 300, {}], ["grad", 100, 300, {"sums": 1}], ["grad", 100, 300, {"sums": 1, "gate": 30}],
                           ["grad", 100, 300, {"sums": 1, "gate": 100}], ["grad", 100, 4096, {"sums": 1}], ["grad", 1360, 4096, {"sums": 1}],
                           ["grad", 1361, 4096, {"sums": 1}], ["grad", 100, 4097, {"sums": 1}], ["grad", 0, 300, {"sums": 1}],
                           ["grad", 300, 300, {"sums": 1, "gate": 1}], ["grad", 544, 300, {"sums": 1, "gate": 272}],
                           ["norm", 0, 300, {"col": 1}]])
    sums, apart = ["residual_grad", "column_grad"], ["residual_grad", "column_sums", "column_grad"]
    assert [[n.rstrip("_") for n in g] for g in got] == [["block_cast"], [], ["residual_norm"], ["residual_norm", "block_cast"], ["residual_grad"],
                                                         sums, sums, sums, apart, apart, sums, sums, ["column_grad"],
                                                         sums + ["post_grad"], sums + ["post_grad"], []]


def grids(qe, hip, cases):
    got = []
    for kind, *args in cases:
        hip.clear()
        if kind == "product":
            m, n, k = args
            a, b = (qe.make_blocked(ADDR, (k + 15) // 16 * 16, ADDR, (k + 511) // 512 * 4, 0, rows) for rows in (1, 128))
            st = qe.qe_fp8_gemm_block(a, b, m, n, k, None, ADDR, qe.BF16, n, stream=0)
        else:
            rows, cols, gate_rows = args
            ms = [qe.make_matrix(i * ADDR, cols, qe.BF16) for i in range(1, 7)]
            d = qe.make_residual(post_norm=True, post_weight=ADDR, pre_norm=True, pre_weight=ADDR, gate=ADDR, ld_gate=cols, gate_rows=gate_rows)
            st = qe.qe_residual_norm_grad(*ms[:4], rows, cols, d, ADDR, ADDR, *ms[4:], ADDR, 2 * ADDR, 3 * ADDR, qe.INIT, ADDR, stream=0)
        assert st == "OK", st
        got.append([[w[2], int(w[3].split("=")[1])] for w in hip.log("launch")])
    return got


@pytest.mark.parametrize("units", [64, 256])
def test_products_get_their_kernels(units, monkeypatch):
    """Blocks of 16 x 16 up to 16 rows, or where they fill the units once after 1025 (twice after 12289) columns; else tiles."""
    monkeypatch.setenv("FAKE_HIP_UNITS", str(units))
    n = units
    got = calls(grids, [["product", m, nn, k] for m, nn, k in ((16, 64 * n, 128), (256, n, 1025), (257, n, 1025), (256, n, 1024), (512, n, 12289),
                                                               (513, n, 12289), (8192, 8192, 8192))])
    assert ["block_rows_kernel" in g[0][0] for g in got] == [True, True, False, False, True, False, False]
    assert "block_large_kernel" in got[-1][0][0] and "block_ring_kernel" in got[2][0][0]


def test_launches_hold_less_than_2_to_32_lanes():
    """Kernels with 512 lanes a workgroup (rows of products) and 1024 (sums of columns) at the largest sizes that are accepted."""
    got = calls(grids, [["product", 16, (1 << 27) - 16, 2048], ["product", 16, 1 << 27, 2048], ["product", 1, (1 << 29) - 32, 128],
                        ["grad", (1 << 22) - 1, 8192, 1], ["grad", (1 << 22) - 1, 16384, 1], ["grad", 8 * 272, 256, 272], ["grad", 8 * 256, 256, 256],
                        ["grad", 257 * 16, 256, 16]])
    assert "block_rows_kernel" in got[0][0][0] and got[0][0][1] == (1 << 23) - 1
    assert "block_rows_kernel" not in got[1][0][0] and got[2][0][1] * 256 < 1 << 32
    for g in got[3:5]:
        assert [n for n, _ in g if "column_grad" in n] and all(w * 1024 < 1 << 32 for _, w in g)
    assert [[w for n, w in g if "column_grad" in n] for g in got[5:]] == [
        [4 + 8 * 4], [4 + 4], [4 + 65]]  # groups of 17 chunks, of 16: together, a wave each; more than 256 groups: sixteen a workgroup


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
    src = ('#include <stdio.h>\n#include "qe.h"\nint main(void) { printf("%zu %zu %zu\\n", sizeof(qe_blocked), sizeof(qe_matrix), '
           'sizeof(qe_residual)); return 0; }\n')
    with tempfile.TemporaryDirectory() as td:
        c, exe = os.path.join(td, "s.c"), os.path.join(td, "s")
        open(c, "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), c, "-o", exe], check=True)
        got = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in got] == [ctypes.sizeof(t) for t in (qe.Blocked, qe.Matrix, qe.Residual)]
