"""A product's residual at its output's own address, on the host: accumulated in place where both lie alike, else refused (a
tile's stores would change residual values that another tile has yet to read)."""
import pytest

from tests.fake_hip import ADDR, calls
from tests.libqe import need_lib

M, N, K = 300, 520, 256
FAR = 2 * ADDR


def product(qe, kind, residual, residual_dtype, ld_residual, c_dtype, ldc, m=M):
    epi = qe.make_epilogue(residual=residual, residual_dtype=residual_dtype, ld_residual=ld_residual)
    if kind == "act":
        return qe.qe_fp8_gemm_act(ADDR, 0, K, ADDR, 0, K, m, N, K, ADDR, ADDR, epi, ADDR, c_dtype, ldc, stream=0)
    op = qe.make_blocked(ADDR, K, ADDR, 4, 0)
    return qe.qe_fp8_gemm_block(op, op, m, N, K, epi, ADDR, c_dtype, ldc, stream=0)


def statuses(qe, hip, kind, cases):
    return [product(qe, kind, *c) for c in cases]


@pytest.mark.parametrize("kind", ["act", "block"])
def test_a_residual_in_place_lies_as_the_output(kind):
    qe = need_lib()
    f32, bf16 = qe.F32, qe.BF16
    refused = [(ADDR, bf16, N, f32, N), (ADDR, f32, N, bf16, N), (ADDR, bf16, N + 8, bf16, N), (ADDR, f32, N, f32, N + 1),
               (ADDR, bf16, 2 * N, f32, N),  # rows at the same bytes, elements not
               (ADDR, bf16, N, f32, N, 1)]
    taken = [(ADDR, f32, N, f32, N), (ADDR, bf16, N + 3, bf16, N + 3),
             (ADDR, bf16, N, bf16, N + 8, 1),  # one row: no stride is used
             (ADDR, bf16, N, f32, N, 0),       # nothing to write
             (FAR, bf16, N + 8, f32, N), (0, bf16, N, f32, N)]
    assert calls(statuses, kind, refused) == ["INVALID_ARG"] * len(refused)
    assert calls(statuses, kind, taken) == ["OK"] * len(taken)
