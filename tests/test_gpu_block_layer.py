"""A residual block's linear with block scales, forward and backward, as one sequence of calls: the norms write the FP8 codes
that the products read, and the products' output is what the norms' gradient reads.

Each step is held against float64 of what the calls before it stored, so a step's tolerance is its own: products 1e-3 of
their largest value, as for random codes in test_gpu_blocks.py, and half an ulp of BF16 (2^-8) where that is stored; sums and
gradients of the norms as in test_gpu_residual_norm.py (u = 2^-24; 200 u of the terms' magnitudes, a column sum of R rows
R / 4 more).
"""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import fp8
from tests.gpu_util import dev, torch
from tests.libqe import need_lib
from tests.test_gpu_activation import U
from tests.test_gpu_residual_norm import host, within

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-3))
SHAPES = [(1, 128, 64), (33, 648, 200), (300, 1000, 520), (1040, 4096, 257)]


class Codes:
    """Codes as the products want them."""

    def __init__(self, qe, rows, cols, fmt, block_rows, d):
        self.rows, self.cols, self.fmt, self.br = rows, cols, fmt, block_rows
        self.q = torch.full((rows, -(-cols // 16) * 16), 0x3A, dtype=torch.uint8, device=d)
        self.e = torch.full((-(-rows // block_rows), -(-cols // 512) * 4), 200, dtype=torch.uint8, device=d)
        self.h = qe.make_blocked(self.q, self.q.stride(0), self.e, self.e.stride(0), fmt, block_rows)

    def values(self):
        q, e = self.q[:, :self.cols].cpu().numpy(), self.e[:, :-(-self.cols // 128)].cpu().numpy()
        return ob.unpack(q, e, ("E4M3", "E5M2")[self.fmt], self.br)


class Layer:
    def __init__(self, qe, d, tokens, hidden, out, seed, gate_rows=128):
        self.qe, self.sizes, self.gate_rows = qe, (tokens, hidden, out), gate_rows
        g = torch.Generator(device=d)
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(s, device=d, generator=g)  # noqa: E731
        bf = lambda *s: rnd(*s).bfloat16()  # noqa: E731
        groups = -(-tokens // gate_rows)
        self.x, self.y, self.dr, self.dz = bf(tokens, hidden), bf(tokens, hidden), bf(tokens, hidden), bf(tokens, out)
        self.w, self.post_w, self.pre_w = bf(out, hidden) * 0.05, 1 + 0.1 * rnd(hidden), 1 + 0.1 * rnd(hidden)
        self.gate = rnd(groups, hidden)
        zero = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device=d)  # noqa: E731
        self.r, self.dh, self.dx, self.dy = (zero(tokens, hidden, t=torch.bfloat16) for _ in range(4))
        self.z, self.dw = zero(tokens, out, t=torch.bfloat16), zero(out, hidden)
        self.f1, self.f2, self.dpost, self.dpre, self.dgate = zero(tokens), zero(tokens), zero(hidden), zero(hidden), zero(groups, hidden)
        self.ws = zero(2 * hidden * groups * -(-min(gate_rows, tokens) // 16))
        c = lambda rows, cols, fmt, br: Codes(qe, rows, cols, fmt, br, d)  # noqa: E731
        self.h_row, self.h_col = c(tokens, hidden, 0, 1), c(hidden, tokens, 0, 1)
        self.w_row, self.w_col = c(out, hidden, 0, 128), c(hidden, out, 0, 128)
        self.dz_row, self.dz_col = c(tokens, out, 1, 1), c(out, tokens, 1, 1)
        self.desc = qe.make_residual(0.875, 0.5, True, self.post_w, EPS, True, self.pre_w, EPS, qe.F32, 0.0, self.gate, qe.F32, hidden, gate_rows)
        self.outs = [self.r, self.z, self.dw, self.dh, self.dx, self.dy, self.dpost, self.dpre, self.dgate, self.f1, self.f2]

    def m(self, t):
        return self.qe.make_matrix(t, t.stride(0), self.qe.BF16)

    def step(self):
        """dw is increased, the rest written."""
        qe, (t, h, o), m = self.qe, self.sizes, self.m
        epi = qe.make_epilogue(residual=self.dw, residual_dtype=qe.F32, ld_residual=h)
        for st in (qe.qe_quantize_fp8_block(m(self.w), o, h, self.w_row.h, self.w_col.h),
                   qe.qe_residual_norm(m(self.x), m(self.y), t, h, self.desc, m(self.r), None, self.h_row.h, self.h_col.h, self.f1, self.f2),
                   qe.qe_fp8_gemm_block(self.h_row.h, self.w_row.h, t, o, h, None, self.z, qe.BF16, o),
                   qe.qe_quantize_fp8_block(m(self.dz), t, o, self.dz_row.h, self.dz_col.h),
                   qe.qe_fp8_gemm_block(self.dz_row.h, self.w_col.h, t, h, o, None, self.dh, qe.BF16, h),
                   qe.qe_fp8_gemm_block(self.dz_col.h, self.h_col.h, o, h, t, epi, self.dw, qe.F32, h),
                   qe.qe_residual_norm_grad(m(self.dr), m(self.dh), m(self.r), m(self.y), t, h, self.desc, self.f1, self.f2, m(self.dx), m(self.dy),
                                            self.dpost, self.dpre, self.dgate, qe.INIT, self.ws)):
            assert st == "OK", st


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_backward(shape):
    c = Layer(need_lib(), dev(), *shape, 1)
    c.step()
    torch.cuda.synchronize()
    x, y, r, dr, dh = (host(t) for t in (c.x, c.y, c.r, c.dr, c.dh))
    opt = dict(x_scale=0.875, y_scale=0.5, post=host(c.post_w), post_eps=EPS, gate=host(c.gate), gate_rows=c.gate_rows)
    branch = np.abs(ob.residual(None, y, **opt))
    within(r, ob.residual(x, y, **opt), 34 * U * branch + 4 * U * np.abs(x), True)
    h, w, dz = ob.norm(r, EPS, host(c.pre_w)), host(c.w), host(c.dz)
    for codes, v in ((c.h_row, h), (c.h_col, h.T), (c.w_row, w), (c.w_col, w.T), (c.dz_row, dz), (c.dz_col, dz.T)):
        # half a step of the code: 2^-4 or 2^-3 of the value, of subnormal codes 2^-10 / 224 or 2^-17 / 28672 of their block's largest value
        half, low = ((2.0 ** -4, 2.0 ** -17), (2.0 ** -3, 2.0 ** -31))[codes.fmt]
        assert (np.abs(codes.values() - v) <= np.maximum(half * np.abs(v), low * np.abs(v).max()) * (1 + 1e-4) + 1e-37).all()
    for got, a, b, bf16 in ((c.z, c.h_row, c.w_row, True), (c.dh, c.dz_row, c.w_col, True), (c.dw, c.dz_col, c.h_col, False)):
        want = a.values() @ b.values().T
        within(host(got), want, 1e-3 * np.abs(want).max(), bf16)
    want = ob.residual_grad(dr, dh, r, y, pre=host(c.pre_w), pre_eps=EPS, **opt)
    f, g = ob.rstd(r, EPS)[:, None], ob.rstd(y, EPS)[:, None]
    n, m, pw, ow = np.abs(r) * f, np.abs(y) * g, np.abs(host(c.pre_w)), np.abs(host(c.post_w))
    gate = np.abs(np.repeat(host(c.gate), min(c.gate_rows, shape[0]), 0)[:shape[0]])
    t = np.abs(dr) + f * (np.abs(dh) * pw + n * (np.abs(dh) * pw * n).mean(1, keepdims=True))
    b = 0.5 * t * gate * ow
    u = (200 + shape[0] / 4) * U
    within(host(c.dx), want["dx"], 200 * U * t, True)
    within(host(c.dy), want["dy"], 200 * U * g * (b + m * (b * m).mean(1, keepdims=True)), True)
    within(host(c.dpre), want["dpre"], u * (np.abs(dh) * n).sum(0), False)
    within(host(c.dpost), want["dpost"], u * (0.5 * t * gate * m).sum(0), False)
    rows = np.arange(shape[0]) // c.gate_rows
    within(host(c.dgate), want["dgate"], u * np.stack([(0.5 * t * m * ow)[rows == i].sum(0) for i in range(c.gate.shape[0])]), False)


def test_two_graphs_and_two_streams():
    """Two layers captured apart and replayed on new inputs, between eager steps of both on streams of their own at once."""
    qe, d = need_lib(), dev()
    layers = [Layer(qe, d, *s, i) for i, s in enumerate(((300, 1000, 520), (70, 4096, 200)))]
    graphs = []
    for c in layers:
        c.step()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.step()
    streams = [torch.cuda.Stream() for _ in layers]
    for i in range(4):
        for c in layers:
            for t in (c.x, c.y, c.dr, c.dz, c.w):
                t.mul_(-1.25)
            c.ws.fill_(float("nan"))
            c.dw.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in c.outs] for c in layers]
        for c in layers:
            for t in c.outs:
                t.zero_()
        torch.cuda.synchronize()
        for c, s in zip(layers, streams):
            with torch.cuda.stream(s):
                c.step()
        torch.cuda.synchronize()
        for c, was in zip(layers, got):
            assert all(torch.equal(a, b) for a, b in zip(was, c.outs)), i
