"""The norms around a residual sum and their gradient on the GPU, against float64.

With u = 2^-24.  A mean of squares of up to 16384 values adds at most 16 terms in a lane and 6 + 16 across lanes, all
positive: relative error below 40 u, half of that in 1 / sqrt, which adds two roundings: 24 u.  A value of p, h has four
more roundings: 32 u of it; r two more of either term.  A stored value adds half an ulp of BF16, 2^-8 of it.  h is held
against the norm of r as the call stored it.  Gradients: every term of t = dr + f (d - n mean(d n)) is within 100 u of
its magnitude (two sums like those above, one of them of signed terms, whose magnitudes then count), dy's within 100 u
of its own on top, and a column's sum of R rows adds at most R / 4 + 40 roundings of its terms' magnitudes.
"""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import fp8
from tests.gpu_util import dev, torch
from tests.libqe import need_lib
from tests.test_gpu_activation import FMTS, U, filled, untouched
from tests.test_gpu_blocks import T, Blocks, dtype, matrix

pytestmark = pytest.mark.gpu
EPS = 1e-3
ids = lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else None  # noqa: E731


def host(t):
    return None if t is None else t.double().cpu().numpy()


def within(got, want, tol, bf16):
    tol = tol + np.abs(want) * (2.0 ** -8 + 2.0 ** -18) * bf16 + 1e-37
    off = np.abs(got - want) - tol
    assert np.isfinite(got).all() and off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))


class Case:
    """Inputs of one call; kw: x, y, r, h: types ("f32", "bf16" or None), post, pre: norms, weights ("f32", "bf16" or None),
    gate_rows (0: no gate), xs, ys, offset, pad."""

    def __init__(self, qe, d, rows, cols, seed, x="bf16", y="bf16", r="bf16", h=None, post=True, pre=True, weights="bf16", gate_rows=0,
                 xs=1.0, ys=1.0, offset=0.0, pad=0):
        self.__dict__.update(qe=qe, d=d, rows=rows, cols=cols, kinds=dict(x=x, y=y, r=r, h=h), post=post, pre=pre, xs=xs, ys=ys, pad=pad,
                             offset=offset, gate_rows=gate_rows)
        rng = np.random.default_rng(seed)
        self.rng = rng

        def put(kind, values):
            if kind is None:
                return None
            t = filled(values.shape[0], values.shape[1] + pad, T[kind], d)
            t[:values.shape[0], :values.shape[1]] = torch.from_numpy(values).to(d)
            return t
        self.put = put
        size = np.exp(rng.normal(size=(rows, 1)))
        self.x, self.y = put(x, rng.normal(size=(rows, cols)) * size), put(y, rng.normal(size=(rows, cols)) * 3.0)
        w = lambda: None if weights is None else torch.from_numpy(1.0 - offset + 0.2 * rng.normal(size=cols)).to(d).to(T[weights])  # noqa: E731
        self.post_w, self.pre_w = w(), w()
        groups = -(-rows // gate_rows) if gate_rows else 0
        self.gate = put("f32", rng.normal(size=(groups, cols))) if groups else None
        self.groups = groups
        wdt = qe.F32 if weights is None else dtype(qe, T[weights])
        self.desc = qe.make_residual(xs, ys, post, self.post_w, EPS, pre, self.pre_w, EPS, wdt, offset, self.gate, qe.F32, cols + pad, gate_rows)
        # the same in float64
        eff = lambda t: None if t is None else host(t) + np.float64(np.float32(offset))  # noqa: E731
        self.opt = dict(x_scale=float(np.float32(xs)), y_scale=float(np.float32(ys)), post=eff(self.post_w), post_eps=float(np.float32(EPS)) if post else None,
                        gate=None if self.gate is None else host(self.gate[:groups, :cols]), gate_rows=max(gate_rows, 1))
        self.pre_eff, self.pre_eps = eff(self.pre_w), float(np.float32(EPS))

    def values(self, t):
        return None if t is None else host(t[:self.rows, :self.cols])

    def handle(self, t):
        return matrix(self.qe, t)

    def forward(self, row=None, col=None, in_place=False):
        rows, cols, d = self.rows, self.cols, self.d
        xv, yv = self.values(self.x), self.values(self.y)
        out = lambda k: None if k is None else filled(rows, cols + self.pad, T[k], d)  # noqa: E731
        self.r = self.x if in_place else out(self.kinds["r"])
        self.h = out(self.kinds["h"])
        self.post_rstd = torch.full((rows + 1,), 77.0, device=d) if self.post and self.y is not None else None
        self.pre_rstd = torch.full((rows + 1,), 77.0, device=d) if self.pre else None
        self.row = Blocks(self.qe, rows, cols, row, 1, d, self.pad) if row is not None else None
        self.col = Blocks(self.qe, cols, rows, col, 1, d, self.pad) if col is not None else None
        st = self.qe.qe_residual_norm(self.handle(self.x), self.handle(self.y), rows, cols, self.desc, self.handle(self.r), self.handle(self.h),
                                      self.row.h if self.row else None, self.col.h if self.col else None, self.post_rstd, self.pre_rstd)
        assert st == "OK"
        torch.cuda.synchronize()
        return xv, yv

    def check_forward(self, xv, yv):
        want = ob.residual(xv, yv, **self.opt)
        branch = 0.0 if yv is None else np.abs(ob.residual(None, yv, **self.opt))
        tol = 34 * U * branch + 4 * U * (0.0 if xv is None else np.abs(self.opt["x_scale"] * xv))
        if self.post_rstd is not None:
            within(host(self.post_rstd[:self.rows]), ob.rstd(yv, self.opt["post_eps"]), 24 * U * ob.rstd(yv, self.opt["post_eps"]), False)
            assert float(self.post_rstd[self.rows]) == 77
        r = want
        if self.r is not None:
            r = self.values(self.r)
            within(r, want, tol, self.r.dtype == torch.bfloat16)
            assert untouched(self.r, self.rows, self.cols)
            tol = 0.0
        if not self.pre:
            return
        f = ob.rstd(r, self.pre_eps)
        within(host(self.pre_rstd[:self.rows]), f, 24 * U * f + (0 if self.r is not None else 100 * U * f), False)
        assert float(self.pre_rstd[self.rows]) == 77
        h = ob.norm(r, self.pre_eps, self.pre_eff)
        w = 1.0 if self.pre_eff is None else np.abs(self.pre_eff)
        tol = tol * f[:, None] * w + 32 * U * np.abs(h) + (0 if self.r is not None else 100 * U * np.abs(h))
        if self.h is not None:
            within(self.values(self.h), h, tol, self.h.dtype == torch.bfloat16)
            assert untouched(self.h, self.rows, self.cols)
        for b, v, t in ((self.row, h, tol), (self.col, h.T, np.broadcast_to(tol, h.shape).T)):
            if b is None:
                continue
            q, e = b.get()
            name = FMTS[b.fmt]
            step = np.repeat(2.0 ** (e.astype(np.float64) - 127), 128, 1)[:, :b.cols]
            half = {"E4M3": 2.0 ** -4, "E5M2": 2.0 ** -3}[name]
            low = {"E4M3": 2.0 ** -10, "E5M2": 2.0 ** -17}[name]
            off = np.abs(fp8.decode(q, name) * step - v) - (np.maximum(half * np.abs(v), low * step) + 2 * t)
            assert off.max() <= 0, off.max()
            top = np.maximum.reduceat(np.abs(v), np.arange(0, b.cols, 128), axis=1) / 2.0 ** (e.astype(np.float64) - 127)
            fmax = {"E4M3": 448.0, "E5M2": 57344.0}[name]
            assert ((top <= fmax * (1 + 1e-5)) & ((top > fmax / 2 * (1 - 1e-5)) | (e == 1))).all()
            assert untouched(b.q, b.rows, b.cols) and untouched(b.e, *b.groups)


FORMS = [dict(), dict(r="f32", x="f32", y="f32", h="f32", weights="f32", pad=1), dict(h="bf16", gate_rows=1 << 40, xs=0.875, ys=0.5),
         dict(x="f32", r="f32", h="bf16", gate_rows=3, offset=1.0, pad=3), dict(post=False, gate_rows=1, ys=0.22, h="f32"), dict(pre=False, weights=None),
         dict(x=None, h="bf16", weights=None), dict(y=None, r=None, h="bf16", pad=5), dict(y=None, xs=2.0, h="f32"), dict(r=None, h="f32", x="f32", y="f32")]
SHAPES = [(1, 1), (1, 7), (3, 128), (5, 130), (17, 512), (2, 513), (33, 1000), (3, 2730), (2, 8192), (2, 8193), (1, 16384), (2, 12345)]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(f"{k}{v}" for k, v in f.items()) or "plain")
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_forward(shape, form):
    c = Case(need_lib(), dev(), *shape, sum(shape), **form)
    codes = form.get("pre", True)
    c.check_forward(*c.forward(row=0 if codes else None, col=0 if codes and (c.kinds["r"] or (c.y is None and c.xs == 1.0)) else None))


@pytest.mark.parametrize("shape", [(1, 300), (130, 264), (300, 1000), (257, 4099)], ids=ids)
@pytest.mark.parametrize("fmt", [0, 1], ids=FMTS)
def test_codes_are_the_casts_of_h(shape, fmt):
    """Row-wise and transposed codes are, bit for bit, what the block cast makes of the FP32 h."""
    qe, d = need_lib(), dev()
    c = Case(qe, d, *shape, 3, x="bf16", r="bf16", h="f32", gate_rows=7, pad=1)
    c.check_forward(*c.forward(row=fmt, col=fmt))
    row, col = Blocks(qe, *shape, fmt, 1, d, 1), Blocks(qe, *shape[::-1], fmt, 1, d, 1)
    assert qe.qe_quantize_fp8_block(matrix(qe, c.h), *shape, row.h, col.h) == "OK"
    torch.cuda.synchronize()
    for a, b in ((c.row, row), (c.col, col)):
        assert torch.equal(a.q, b.q) and torch.equal(a.e, b.e)


def test_the_stream_in_place():
    """r over x, and h over y."""
    for shape in ((3, 300), (130, 1000)):
        c = Case(need_lib(), dev(), *shape, 4, gate_rows=2, xs=0.5)
        c.check_forward(*c.forward(row=0, col=0, in_place=True))
        a = Case(need_lib(), dev(), *shape, 5, h="bf16")
        b = Case(need_lib(), dev(), *shape, 5, h="bf16")
        a.forward()
        assert b.qe.qe_residual_norm(b.handle(b.x), b.handle(b.y), *shape, b.desc, b.handle(b.x), b.handle(b.y)) == "OK"
        assert torch.equal(a.r, b.x) and torch.equal(a.h, b.y)


def test_zero_rows_and_rows_with_nan_or_infinity():
    """A zero row gives zeros (a padded batch); a NaN or an infinity spoils its own row alone."""
    qe, d = need_lib(), dev()
    c = Case(qe, d, 6, 300, 1, h="f32", r="f32")
    for t in (c.x, c.y):
        t[1, :300] = 0
    c.x[2, 5], c.y[4, 299] = float("nan"), float("inf")
    c.forward(row=0)
    assert bool((c.r[1, :300] == 0).all()) and bool((c.h[1, :300] == 0).all()) and bool(((c.row.q[1, :300] & 0x7F) == 0).all())
    assert c.row.e[1, :3].tolist() == [1, 1, 1]
    for i in (2, 4):
        assert bool(c.h[i, :300].isnan().all()) and bool((c.row.e[i, :3] == 255).all())
    fine = [0, 1, 3, 5]
    assert bool(c.h[fine, :300].isfinite().all()) and bool((c.row.e[fine, :3] < 255).all())


# ------------------------------------------------------------------ gradient
def check_grad(c, use_dr=True, use_dh=True, dt="bf16", out="bf16", sums=True, mode=0, in_place=False):
    qe, d, rows, cols, pad = c.qe, c.d, c.rows, c.cols, c.pad
    c.forward()
    dr = c.put(dt, c.rng.normal(size=(rows, cols)) * 0.01) if use_dr else None
    dh = c.put(dt, c.rng.normal(size=(rows, cols)) * 0.01) if use_dh else None
    stream = c.r if c.r is not None else c.x
    drv, dhv, rv, yv = (c.values(t) for t in (dr, dh, stream, c.y))
    dx = dr if in_place else filled(rows, cols + pad, T[out], d)
    dy = None if c.y is None else (dh if in_place else filled(rows, cols + pad, T[out], d))
    vec = lambda *s: torch.full(s, 3.0, device=d)  # noqa: E731
    post = vec(cols + 1) if sums and c.post and c.y is not None and c.post_w is not None else None
    pre = vec(cols + 1) if sums and use_dh and c.pre_w is not None else None
    gate = vec(c.groups + 1, cols + pad) if sums and c.gate is not None and c.y is not None else None
    gr = min(c.gate_rows or rows, rows)
    ws = torch.full((2 * cols * max(c.groups, 1) * -(-gr // 16) + 1,), 5.0, device=d) if sums else None
    if ws is not None:
        ws[:-1] = float("nan")
    st = qe.qe_residual_norm_grad(c.handle(dr), c.handle(dh), c.handle(stream), c.handle(c.y), rows, cols, c.desc, c.post_rstd, c.pre_rstd,
                                  c.handle(dx), c.handle(dy), post, pre, gate, mode, ws, cols + pad)
    assert st == "OK"
    torch.cuda.synchronize()
    want = ob.residual_grad(drv, dhv, rv, yv, pre=c.pre_eff, pre_eps=c.pre_eps, **c.opt)
    # magnitudes of what each value is a sum of
    t = 0.0 if drv is None else np.abs(drv)
    if dhv is not None:
        f = ob.rstd(rv, c.pre_eps)[:, None]
        n, w = np.abs(rv) * f, 1.0 if c.pre_eff is None else np.abs(c.pre_eff)
        t = t + f * (np.abs(dhv) * w + n * (np.abs(dhv) * w * n).mean(1, keepdims=True))
    xs, ys = abs(c.opt["x_scale"]), abs(c.opt["y_scale"])
    bf = out == "bf16" or (in_place and dt == "bf16")
    within(c.values(dx), want["dx"], 100 * U * xs * t, bf)
    assert untouched(dx, rows, cols)
    more = rows / 4 + 40
    plus = 3.0 if mode else 0.0
    if pre is not None:
        within(host(pre[:cols]), want["dpre"] + plus, (30 + more) * U * (np.abs(dhv) * n).sum(0) + 8 * U * plus, False)
        assert float(pre[cols]) == 3
    if yv is not None:
        m = np.abs(yv) if not c.post else np.abs(yv) * ob.rstd(yv, EPS)[:, None]
        w = 1.0 if c.opt["post"] is None or not c.post else np.abs(c.opt["post"])
        g = 1.0 if c.opt["gate"] is None else np.abs(np.repeat(c.opt["gate"], c.opt["gate_rows"] if c.opt["gate_rows"] < rows else rows, 0)[:rows])
        b = ys * t
        mag = b * g
        if c.post:
            mag = ob.rstd(yv, EPS)[:, None] * (mag * w + m * (mag * w * m).mean(1, keepdims=True))
        within(c.values(dy), want["dy"], 200 * U * mag, bf)
        assert untouched(dy, rows, cols)
        if post is not None:
            within(host(post[:cols]), want["dpost"] + plus, (150 + more) * U * (b * g * m).sum(0) + 8 * U * plus, False)
            assert float(post[cols]) == 3
        if gate is not None:
            mags = np.stack([(b * m * w)[i * gr:(i + 1) * gr].sum(0) for i in range(c.groups)])
            within(host(gate[:c.groups, :cols]), want["dgate"] + plus, (150 + more) * U * mags + 8 * U * plus, False)
            assert bool((gate[c.groups] == 3).all()) and bool((gate[:, cols:] == 3).all())
    if ws is not None:
        assert float(ws[-1]) == 5
    return dx, dy, post, pre, gate


GRAD_FORMS = [dict(), dict(r="f32", x="f32", y="f32", weights="f32", pad=1), dict(gate_rows=1 << 40, xs=0.875, ys=0.5), dict(gate_rows=3, offset=1.0, pad=3),
              dict(post=False, gate_rows=1, ys=0.22), dict(post=False), dict(weights=None, gate_rows=20), dict(y=None, r=None, pad=5), dict(r="f32", y="bf16")]
GRAD_SHAPES = [(1, 1), (1, 7), (3, 128), (17, 512), (33, 513), (16, 1000), (100, 2730), (2, 8192), (35, 8193), (5, 16384), (300, 70),
               (700, 4104), (40, 4103), (1400, 2600), (600, 1100)]  # columns summed with the rows, or by a kernel of their own


@pytest.mark.parametrize("form", GRAD_FORMS, ids=lambda f: "-".join(f"{k}{v}" for k, v in f.items()) or "plain")
@pytest.mark.parametrize("shape", GRAD_SHAPES, ids=ids)
def test_gradient(shape, form):
    c = Case(need_lib(), dev(), *shape, sum(shape) + 1, **form)
    dt = "f32" if form.get("x") == "f32" else "bf16"
    check_grad(c, dt=dt, out=dt)


@pytest.mark.parametrize("how", [dict(use_dr=False), dict(use_dh=False), dict(sums=False), dict(mode=1), dict(in_place=True), dict(out="f32"), dict(dt="f32")],
                         ids=lambda h: "-".join(f"{k}{v}" for k, v in h.items()))
@pytest.mark.parametrize("form", [dict(gate_rows=30), dict(post=False, weights="f32", pad=1)], ids=["gate", "one_norm"])
def test_gradient_options(form, how):
    for shape in ((70, 300), (18, 9000)):
        check_grad(Case(need_lib(), dev(), *shape, 8, **form), **how)


@pytest.mark.parametrize("shape,gate_rows", [((8704, 70), 1088), ((600, 200), 2), ((257, 64), 1), ((1028, 130), 4), ((4096, 520), 16), ((2176, 64), 272)],
                         ids=ids)
def test_gradient_of_many_groups_and_chunks(shape, gate_rows):
    """Groups of more than 16 chunks, more than 256 groups, and 256 of one chunk."""
    check_grad(Case(need_lib(), dev(), *shape, 9, gate_rows=gate_rows, weights="f32"))
    check_grad(Case(need_lib(), dev(), *shape, 10, gate_rows=gate_rows, weights="f32", post=False), mode=1)


def test_no_rows():
    """Nothing but the weights' gradients, which INIT clears and ACCUM keeps."""
    qe, d = need_lib(), dev()
    m = qe.make_matrix(torch.zeros(8, device=d), 100, qe.F32)
    w = torch.ones(100, device=d)
    desc = qe.make_residual(post_norm=True, post_weight=w, pre_norm=True, pre_weight=w)
    for mode, left in ((qe.ACCUM, 3.0), (qe.INIT, 0.0)):
        a, b = torch.full((100,), 3.0, device=d), torch.full((100,), 3.0, device=d)
        assert qe.qe_residual_norm_grad(m, m, m, m, 0, 100, desc, w, w, m, m, a, b, None, mode, w) == "OK"
        torch.cuda.synchronize()
        assert bool((a == left).all()) and bool((b == left).all())


@pytest.mark.parametrize("shape", [(300, 264), (20, 8200)], ids=ids)
def test_rows_of_long_strides(shape):
    """Rows so far apart that elements are past 2^31: the bits of the same calls on packed rows."""
    qe, d = need_lib(), dev()
    rows, cols = shape
    ld = 2 ** 32 // rows + 7
    g = torch.Generator(device=d)
    g.manual_seed(4)
    w, groups = torch.randn(cols, device=d, generator=g), -(-rows // 7)
    gate = torch.randn((groups, cols), device=d, generator=g)
    packed = [torch.randn(shape, device=d, generator=g).bfloat16() for _ in range(4)]  # x, y, dr, dh
    got = []
    for far in (False, True):
        new = lambda: torch.empty((rows, ld), dtype=torch.bfloat16, device=d) if far else torch.empty(shape, dtype=torch.bfloat16, device=d)  # noqa: E731
        ins = []
        for t in packed:
            ins.append(new())
            ins[-1][:, :cols] = t
        x, y, dr, dh = ins
        r, h = new(), new()
        f1, f2 = torch.zeros(rows, device=d), torch.zeros(rows, device=d)
        sums = [torch.zeros(cols, device=d), torch.zeros(cols, device=d), torch.zeros((groups, cols), device=d)]
        ws = torch.zeros(2 * cols * groups, device=d)
        m = lambda t: qe.make_matrix(t, t.stride(0), qe.BF16)  # noqa: E731
        desc = qe.make_residual(1.0, 0.5, True, w, EPS, True, w, EPS, qe.F32, 0.0, gate, qe.F32, cols, 7)
        row, col = Blocks(qe, rows, cols, 0, 1, d), Blocks(qe, cols, rows, 0, 1, d)
        assert qe.qe_residual_norm(m(x), m(y), rows, cols, desc, m(r), m(h), row.h, col.h, f1, f2) == "OK"
        # in the place of dr and dh
        assert qe.qe_residual_norm_grad(m(dr), m(dh), m(r), m(y), rows, cols, desc, f1, f2, m(dr), m(dh), *sums, qe.INIT, ws) == "OK"
        torch.cuda.synchronize()
        got.append([t[:, :cols].clone() for t in (r, h, dr, dh)] + [f1, f2, *sums, row.q, row.e, col.q, col.e])
        del ins, x, y, dr, dh, r, h
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_gradients_repeat_their_bits_and_replay():
    """Captured with the forward and replayed on new inputs between eager calls: every replay gives the eager bits."""
    qe, d = need_lib(), dev()
    rows, cols = 300, 1000
    c = Case(qe, d, rows, cols, 2, h="bf16", gate_rows=40)
    dr, dh = c.put("bf16", c.rng.normal(size=(rows, cols))), c.put("bf16", c.rng.normal(size=(rows, cols)))
    r, h, dx, dy = (filled(rows, cols, torch.bfloat16, d) for _ in range(4))
    f1, f2 = torch.zeros(rows, device=d), torch.zeros(rows, device=d)
    sums = [torch.zeros(cols, device=d), torch.zeros(cols, device=d), torch.zeros((c.groups, cols), device=d)]
    ws = torch.zeros(2 * cols * c.groups * 3, device=d)
    row, col = Blocks(qe, rows, cols, 0, 1, d), Blocks(qe, cols, rows, 0, 1, d)
    hd = c.handle

    def step():
        assert qe.qe_residual_norm(hd(c.x), hd(c.y), rows, cols, c.desc, hd(r), hd(h), row.h, col.h, f1, f2) == "OK"
        assert qe.qe_residual_norm_grad(hd(dr), hd(dh), hd(r), hd(c.y), rows, cols, c.desc, f1, f2, hd(dx), hd(dy), *sums, qe.INIT, ws) == "OK"
    outs = [r, h, dx, dy, f1, f2, *sums, row.q, row.e, col.q, col.e]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in (c.x, c.y, dr, dh):
            t.mul_(-1.25)
        ws.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
