"""A gated feed-forward block in FP8 on one MI355X: a training step and single-token serving.

    python examples/gated_ffn.py [--tokens 4096 --hidden 4096 --ffn 14336]   # Llama-3-8B-shaped by default

    h = silu(x Wg^T) * (x Wu^T)        qe_fp8_gemm_gated, which keeps both pre-activations in 8 bits
    y = h Wd^T + x                     qe_fp8_gemm_act
    dh = dy Wd                         qe_fp8_gemm_tn
    dg, du from dh and the checkpoint  qe_act_grad, straight to the FP8 codes that the next products read
    dx = [dg du] [Wg; Wu], dW = ..     qe_fp8_gemm_tn, the weight gradients into one flat FP32 buffer

Scales are delayed: every tensor is cast with the scale that its earlier amaxes gave it.  Nothing is allocated in a
step, so it can be captured into a graph.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_23536_amd import qe  # noqa: E402


def _ok(status):
    if status != "OK":
        raise RuntimeError(status)


def _check(name, t, rows, cols, *dtypes):
    """The library sees an address: a tensor of another size, type or stride would be misread, or read and written past."""
    if tuple(t.shape) != (rows, cols) or t.dtype not in dtypes or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s: want a contiguous [%d, %d] tensor of %s on the GPU, got %s of %s" % (
            name, rows, cols, " or ".join(str(d) for d in dtypes), list(t.shape), t.dtype))


def _ld(v):
    return (v + 15) // 16 * 16 if v <= 256 else (v + 127) // 128 * 128  # whole lines for long rows


class Role:
    """One tensor's FP8 codes, row-wise and transposed, and its delayed-scaling state.

    With `reads`, another role: codes (row-wise only) and amaxes of its own, cast with that role's scale.
    """

    def __init__(self, rows, cols, fmt, history=16, reads=None):
        self.rows, self.cols, self.fmt = rows, cols, fmt
        self.row = torch.zeros((rows, _ld(cols)), dtype=torch.uint8, device="cuda")
        self.col = torch.zeros((cols, _ld(rows)), dtype=torch.uint8, device="cuda") if reads is None else None
        self.hist = torch.zeros(history, dtype=torch.float32, device="cuda")
        self.scales = torch.ones(3, dtype=torch.float32, device="cuda")  # scale, its inverse, the inverse of the codes' own
        self.accum = torch.zeros(qe.AMAX_LINES * qe.AMAX_STRIDE, dtype=torch.float32, device="cuda")
        scales = self.scales if reads is None else reads.scales
        self.meta = qe.make_meta(self.hist, scales[0:1], scales[1:2], fmt, 0, self.accum)

    @property
    def inv(self):
        return self.scales[2:3]

    def cast(self, x, rows=None):
        dt = qe.BF16 if x.dtype == torch.bfloat16 else qe.F32
        rows = self.rows if rows is None else rows
        _ok(qe.qe_quantize_fp8(x, dt, rows, self.cols, self.meta, self.row, self.row.shape[1], self.col,
                               0 if self.col is None else self.col.shape[1], self.inv))


class GatedFFN:
    """Weights of one block, the buffers of one microbatch of `tokens` and, apart from those, of up to `serve_tokens` served
    together (`tokens` if not given)."""

    def __init__(self, wg_wu, wd, tokens, act=qe.ACT_SILU, serve_tokens=None):
        self.act, self.tokens = act, tokens
        self.ffn, self.hidden = wd.shape[1], wd.shape[0]
        t, f, d = tokens, self.ffn, self.hidden
        _check("wg_wu", wg_wu, 2 * f, d, torch.bfloat16, torch.float32)
        _check("wd", wd, d, f, torch.bfloat16, torch.float32)
        self.wgu_master, self.wd_master = wg_wu, wd
        self.wgu, self.wd = Role(2 * f, d, qe.E4M3), Role(d, f, qe.E4M3)
        self.x, self.h_q = Role(t, d, qe.E4M3), Role(t, f, qe.E4M3)
        self.dy, self.dgu = Role(t, d, qe.E5M2), Role(t, 2 * f, qe.E5M2)
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.h, self.y = torch.zeros((t, f), **bf), torch.zeros((t, d), **bf)
        self.dh, self.dx = torch.zeros((t, f), **bf), torch.zeros((t, d), **bf)
        self.grad = torch.zeros(3 * f * d, dtype=torch.float32, device="cuda")  # dWgu, then dWd
        groups = (f + qe.SAVED_GROUP - 1) // qe.SAVED_GROUP
        self.codes = torch.zeros((2, t, f), dtype=torch.int8, device="cuda")
        self.exps = torch.zeros((2, t, groups), dtype=torch.uint8, device="cuda")
        self.saved = [qe.make_saved(qe.SAVED_I8, self.codes[i], f, self.exps[i], groups) for i in range(2)]
        # served tokens leave no trace in a training step: codes, outputs and amaxes of their own
        self.serve_tokens = n = t if serve_tokens is None else serve_tokens
        self.serve_x, self.serve_h_q = Role(n, d, qe.E4M3, reads=self.x), Role(n, f, qe.E4M3, reads=self.h_q)
        self.serve_h, self.serve_y = torch.zeros((n, f), **bf), torch.zeros((n, d), **bf)

    def refresh(self):
        """After an optimizer step: the weights' codes, and the scales of the next ones."""
        self.wgu.cast(self.wgu_master)
        self.wd.cast(self.wd_master)
        _ok(qe.qe_amax_scale_update([self.wgu.meta, self.wd.meta]))

    def _up(self, x, h, rows, saved):
        f, w = self.ffn, self.wgu
        _ok(qe.qe_fp8_gemm_gated(x.row, x.fmt, x.row.shape[1], w.row, w.row[f:], w.fmt, w.row.shape[1], rows, f, self.hidden,
                                 x.inv, w.inv, w.inv, self.act, h, qe.BF16, f, saved[0], saved[1]))

    def _down(self, h_q, residual, y, rows):
        d, w = self.hidden, self.wd
        _ok(qe.qe_fp8_gemm_act(h_q.row, h_q.fmt, h_q.row.shape[1], w.row, w.fmt, w.row.shape[1], rows, d, self.ffn, h_q.inv,
                               w.inv, qe.make_epilogue(residual=residual, residual_dtype=qe.BF16, ld_residual=d), y, qe.BF16,
                               d))

    def forward(self, x):
        _check("x", x, self.tokens, self.hidden, torch.bfloat16)
        self.x.cast(x)
        self._up(self.x, self.h, self.tokens, self.saved)
        self.h_q.cast(self.h)
        self._down(self.h_q, x, self.y, self.tokens)
        _ok(qe.qe_amax_scale_update([self.x.meta, self.h_q.meta]))
        return self.y

    def serve(self, x):
        """A few tokens, nothing kept for a backward pass and no scale moved: with the scales of the last training step, and
        between a forward and its backward as well as anywhere else."""
        n = x.shape[0]
        if n > self.serve_tokens:
            raise ValueError("%d tokens in buffers for %d" % (n, self.serve_tokens))
        _check("x", x, n, self.hidden, torch.bfloat16)
        self.serve_x.cast(x, n)
        self._up(self.serve_x, self.serve_h, n, (None, None))
        self.serve_h_q.cast(self.serve_h, n)
        self._down(self.serve_h_q, x, self.serve_y, n)
        return self.serve_y[:n]

    @staticmethod
    def _product(a, a_t, b, b_t, m, n, k, inv, out, dtype, ld):
        _ok(qe.qe_fp8_gemm_tn(a, a_t, a.shape[1], b, b_t, b.shape[1], m, n, k, inv[0], inv[1], out, dtype, ld))

    def backward(self, dy):
        t, f, d = self.tokens, self.ffn, self.hidden
        _check("dy", dy, t, d, torch.bfloat16)
        self.dy.cast(dy)
        self._product(self.dy.row, self.dy.fmt, self.wd.col, self.wd.fmt, t, f, d, (self.dy.inv, self.wd.inv), self.dh, qe.BF16, f)
        _ok(qe.qe_act_grad(self.dh, qe.BF16, f, t, f, self.act, self.saved[0], self.saved[1], meta=self.dgu.meta,
                           q_row=self.dgu.row, ld_row=self.dgu.row.shape[1], q_col=self.dgu.col,
                           ld_col=self.dgu.col.shape[1], scale_inv_snapshot=self.dgu.inv))
        self._product(self.dgu.row, self.dgu.fmt, self.wgu.col, self.wgu.fmt, t, d, 2 * f, (self.dgu.inv, self.wgu.inv), self.dx,
                      qe.BF16, d)
        self.dx += dy  # the residual's own gradient
        dwgu, dwd = self.grad[:2 * f * d], self.grad[2 * f * d:]
        self._product(self.dgu.col, self.dgu.fmt, self.x.col, self.x.fmt, 2 * f, d, t, (self.dgu.inv, self.x.inv), dwgu, qe.F32, d)
        self._product(self.dy.col, self.dy.fmt, self.h_q.col, self.h_q.fmt, d, f, t, (self.dy.inv, self.h_q.inv), dwd, qe.F32, f)
        _ok(qe.qe_amax_scale_update([self.dy.meta, self.dgu.meta]))
        return self.dx, dwgu.view(2 * f, d), dwd.view(d, f)


def make(tokens, hidden, ffn, seed=0):
    """A block with random weights, its input and its output's gradient, after two steps that set the scales."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, sigma):
        return (torch.randn(shape, generator=g, device="cuda") * sigma).to(torch.bfloat16)
    block = GatedFFN(normal(2 * ffn, hidden, sigma=0.02), normal(hidden, ffn, sigma=0.02), tokens)
    x, dy = normal(tokens, hidden, sigma=1.0), normal(tokens, hidden, sigma=0.01)
    block.refresh()
    for _ in range(2):
        block.refresh()
        block.forward(x)
        block.backward(dy)
    return block, x, dy


def reference(block, x, dy):
    """y, dx, dWgu, dWd of the same block in 32 bits, without FP8."""
    wgu, wd, x, dy = (t.float() for t in (block.wgu_master, block.wd_master, x, dy))
    g, u = (x @ wgu.t()).split(block.ffn, 1)
    p = torch.sigmoid(g)
    h, dh = g * p * u, dy @ wd
    dgu = torch.cat((dh * u * p * (1 + g * (1 - p)), dh * g * p), 1)
    return h @ wd.t() + x, dgu @ wgu + dy, dgu.t() @ x, dy.t() @ h


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--ffn", type=int, default=14336)
    a = ap.parse_args()
    block, x, dy = make(a.tokens, a.hidden, a.ffn)

    def timed(name, fn, n=20):
        fn()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(n):
            fn()
        torch.cuda.synchronize()
        print("%-34s %9.1f us" % (name, (time.perf_counter() - t) / n * 1e6))
    got = (block.forward(x), *block.backward(dy))
    for name, v, r in zip(("y", "dx", "dWg, dWu", "dWd"), got, reference(block, x, dy)):
        print("%-9s relative difference to FP32 %.3f" % (name, float((v.float() - r).norm() / r.norm())))
    timed("forward, %d tokens" % a.tokens, lambda: block.forward(x))
    timed("backward", lambda: block.backward(dy))
    timed("serve, 1 token", lambda: block.serve(x[:1]))


if __name__ == "__main__":
    main()
