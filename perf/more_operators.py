"""FP8 with a scale for each block of 128, and the norms and the residual sum between two blocks, as a training or serving
program calls them, and their plain forms.

Four kinds of case:

* ``cast``: a tensor to FP8 codes with one power-of-two scale per 128 values of a row (or per 128 x 128 block: weights),
  row-wise for the forward and dI products, transposed (blocks along the rows) for dW.
* ``product``: Y = X W^T, dX = dY W or dW = dY^T X on such codes, with a residual or accumulated into the main gradient.
* ``norm``: r = xs x + ys gate * norm(y), then h = norm(r), dense or straight to the codes that the next product reads.
* ``grad``: the gradients of that: x, y, both norms' weights and the gate.

Inputs are seeded and made on the GPU.  Activations are N(0, 1) with a size of its own for each token and one channel in a
thousand twenty times larger, weights N(0, 0.02), gradients N(0, 0.01) with a size of its own for each token.
"""
import math

import torch

own = False

FMAX = {"e4m3": 448.0, "e5m2": 57344.0}
FEMAX = {"e4m3": 8, "e5m2": 15}
TORCH_FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "bf16": 2}
BLOCK = 128
EPS = 1e-5


def _cast(**kw):
    case = {"op": "cast", "rows": 1, "cols": 1, "dtype": "bf16", "fmt": "e4m3", "block_rows": 1, "transposed": True, "pad": 0}
    case.update(kw)
    return case


def _product(**kw):
    """kind: fwd and dgrad read a weight with 128 x 128 blocks, wgrad two operands with blocks of one row."""
    case = {"op": "product", "kind": "fwd", "m": 1, "n": 1, "k": 1, "fmt_a": "e4m3", "fmt_b": "e4m3", "residual": False,
            "out": "bf16", "pad": 0}
    case.update(kw)
    return case


def _norm(**kw):
    """gate_rows: rows that share a row of gates (0: no gate).  emit: h dense, as row-wise codes, or as both kinds."""
    case = {"op": "norm", "rows": 1, "cols": 1, "dtype": "bf16", "post": True, "gate_rows": 0, "emit": "dense", "offset": 0.0,
            "xs": 1.0, "ys": 1.0, "pad": 0}
    case.update(kw)
    return case


def _grad(**kw):
    case = {"op": "grad", "rows": 1, "cols": 1, "dtype": "bf16", "post": True, "gate_rows": 0, "offset": 0.0, "xs": 1.0,
            "ys": 1.0, "pad": 0}
    case.update(kw)
    return case


def listed():
    return [
        # The activations of a microbatch of the Llama-3-8B-shaped stage, for the forward product and for dW.
        _cast(name="cast_4096x14336", rows=4096, cols=14336),
        # A weight refresh of the Llama-3-70B-shaped stage: one scale per 128 x 128 block, both orders.
        _cast(name="cast_weight_57344x8192", rows=57344, cols=8192, block_rows=128),
        # Ragged fp32 gradients in odd rows.
        _cast(name="cast_1500x4099_f32", rows=1500, cols=4099, dtype="f32", fmt="e5m2", pad=3),
        # The down projection of one token being served, added to the residual stream.
        _product(name="product_1x4096x14336", m=1, n=4096, k=14336, residual=True),
        # A ragged batch of prompt tokens, odd output rows.
        _product(name="product_1000x2730x1365", m=1000, n=2730, k=1365, pad=3),
        # dI of the widest linear of the Llama-3-8B-shaped stage.
        _product(name="product_dgrad_4096x4096x28672", kind="dgrad", m=4096, n=4096, k=28672, fmt_a="e5m2"),
        # dW of its narrowest one, added to gradients that are kept, and reduced between ranks, in 16 bits.
        _product(name="product_wgrad_6144x4096x2048", kind="wgrad", m=6144, n=4096, k=2048, fmt_a="e5m2", residual=True),
        # The down projection of the Llama-3-70B-shaped stage.
        _product(name="product_8192x8192x28672", m=8192, n=8192, k=28672),
        # One served token between two blocks: its sum, its norm and its codes.
        _norm(name="norm_1x8192", rows=1, cols=8192, emit="row"),
        # A training microbatch of the Llama-3-70B-shaped stage: both norms, a gate per channel, codes for forward and dW.
        _norm(name="norm_8192x8192", rows=8192, cols=8192, gate_rows=8192, emit="both", xs=0.875, ys=0.5),
        # Its backward pass.
        _grad(name="grad_8192x8192", rows=8192, cols=8192, gate_rows=8192, xs=0.875, ys=0.5),
        # Five ragged sequences with a row of gates each, fp32, odd rows.
        _grad(name="grad_1000x2730_f32", rows=1000, cols=2730, dtype="f32", gate_rows=200, offset=1.0, pad=3),
    ]


def _log_int(rng, lo, hi, odd=0.4):
    """A size spread over the logarithm of [lo, hi]: any integer, or (more often) a multiple of 64 where that fits."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() >= odd and v >= 96:
        v = (v + 32) // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("cast", "product", "product", "product", "norm", "grad"))
    pad = rng.choice((0, 0, 3, 16))
    if op == "product":
        kind = rng.choice(("fwd", "fwd", "dgrad", "wgrad"))
        while True:
            m = _log_int(rng, 64, 28672) if kind == "wgrad" else rng.choice((1, rng.randint(2, 16), _log_int(rng, 17, 8192),
                                                                              _log_int(rng, 17, 8192)))
            n, k = _log_int(rng, 32, 28672), _log_int(rng, 64, 8192 if kind == "wgrad" else 28672)
            if 2.0 * m * n * k <= 3.8e12 and n * k <= 28672 * 8192 and m * n <= 28672 * 8192:
                break
        return _product(kind=kind, m=m, n=n, k=k, fmt_a="e4m3" if kind == "fwd" else rng.choice(("e5m2", "e5m2", "e4m3")),
                        fmt_b=rng.choice(("e4m3", "e4m3", "e4m3", "e5m2")), residual=rng.random() < 0.5, pad=pad)
    while True:
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 32, 28672 if op == "cast" else 16384)
        if 4096 <= rows * cols <= (8192 * 28672 if op == "cast" else 8192 * 8192):
            break
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "cast":
        return _cast(rows=rows, cols=cols, dtype=dtype, fmt=rng.choice(("e4m3", "e4m3", "e5m2")),
                     block_rows=rng.choice((1, 1, 128)), transposed=rng.random() < 0.7, pad=pad)
    common = {"rows": rows, "cols": cols, "dtype": dtype, "post": rng.random() < 0.7, "offset": rng.choice((0.0, 1.0)),
              "gate_rows": rng.choice((0, rows, rng.randint(max(1, rows // 8), rows))),
              "xs": rng.choice((1.0, 0.875)), "ys": rng.choice((1.0, 0.22)), "pad": pad}
    if op == "norm":
        return _norm(emit=rng.choice(("dense", "row", "both")), **common)
    return _grad(**common)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _values(g, rows, cols, what, dtype="f32", pad=0):
    """[rows, cols] values in rows of cols + pad.  what: x (activations), w (weights), dy (gradients), or n (plain normal)."""
    sigma = {"x": 1.0, "w": 0.02, "dy": 0.01, "n": 1.0}[what]
    x = torch.zeros((rows, cols + pad), dtype=TDT[dtype], device="cuda")
    size = torch.exp(0.5 * torch.randn((rows, 1), generator=g, device="cuda")) if what in ("x", "dy") else None
    channel = torch.ones((1, cols), device="cuda")
    if what == "x":
        channel[torch.rand((1, cols), generator=g, device="cuda") < 0.001] = 20.0
    chunk = max(1, (1 << 27) // cols)  # rows at a time, drawn in fp32 and rounded
    for r in range(0, rows, chunk):
        n = min(chunk, rows - r)
        v = torch.randn((n, cols), generator=g, device="cuda") * (sigma * channel)
        x[r:r + n, :cols] = v if size is None else v * size[r:r + n]
    return x


def _up(v, to):
    return (v + to - 1) // to * to


def _blocks(v):
    """Blocks of 128 along v, and the row stride their exponents are kept at."""
    n = (v + BLOCK - 1) // BLOCK
    return n, _up(n, 4)


def _buffers(rows, cols, fmt, block_rows=1):
    """Codes [rows, cols] in rows of a multiple of 16 bytes, and their exponents in rows of a multiple of 4."""
    return {"q": torch.zeros((rows, _up(cols, 16)), dtype=torch.uint8, device="cuda"),
            "exps": torch.zeros(((rows + block_rows - 1) // block_rows, _blocks(cols)[1]), dtype=torch.uint8, device="cuda"),
            "rows": rows, "cols": cols, "fmt": fmt, "block_rows": block_rows}


def _operand(g, rows, k, fmt, what, block_rows):
    o = _buffers(rows, k, fmt, block_rows)
    x = _values(g, rows, k, what)
    codes, exps = _encode(x, fmt, block_rows)
    o["q"][:, :k] = codes.view(torch.uint8)
    o["exps"][:, :exps.shape[1]] = exps
    return o


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"case": c}
    if c["op"] == "product":
        m, n, k, kind = c["m"], c["n"], c["k"], c["kind"]
        s["a"] = _operand(g, m, k, c["fmt_a"], "x" if kind == "fwd" else "dy", 1)
        s["b"] = _operand(g, n, k, c["fmt_b"], "x" if kind == "wgrad" else "w", 1 if kind == "wgrad" else BLOCK)
        s["d"] = torch.zeros((m, n + c["pad"]), dtype=TDT[c["out"]], device="cuda")
        s["residual"] = None
        if c["residual"] and kind == "wgrad":  # what the seven microbatches before it left there
            s["d"][:, :n] = _values(g, m, n, "n") * (0.05 * math.sqrt(k))
        elif c["residual"]:
            s["residual"] = _values(g, m, n, "x", "bf16", c["pad"])
        return s
    rows, cols, pad, dt = c["rows"], c["cols"], c["pad"], c["dtype"]
    if c["op"] == "cast":
        what = "w" if c["block_rows"] == BLOCK else ("x" if c["fmt"] == "e4m3" else "dy")
        s["x"] = _values(g, rows, cols, what, dt, pad)
        s["row"] = _buffers(rows, cols, c["fmt"], c["block_rows"])
        s["col"] = _buffers(cols, rows, c["fmt"], c["block_rows"]) if c["transposed"] else None
        return s
    weight = lambda: (_values(g, 1, cols, "n").reshape(-1) * 0.1 + (1.0 - c["offset"])).to(TDT[dt])  # noqa: E731
    s["pre_w"] = weight()
    s["post_w"] = weight() if c["post"] else None
    groups = (rows + c["gate_rows"] - 1) // c["gate_rows"] if c["gate_rows"] else 0
    s["gate"] = (_values(g, groups, cols, "n") * 0.1 + 0.5).to(TDT[dt]) if groups else None
    s["y"] = _values(g, rows, cols, "n", dt, pad)
    if c["op"] == "norm":
        s["x"] = _values(g, rows, cols, "x", dt, pad)
        s["r"] = torch.zeros((rows, cols + pad), dtype=TDT[dt], device="cuda")
        s["h"] = torch.zeros((rows, cols + pad), dtype=TDT[dt], device="cuda") if c["emit"] == "dense" else None
        s["row"] = None if c["emit"] == "dense" else _buffers(rows, cols, "e4m3")
        s["col"] = _buffers(cols, rows, "e4m3") if c["emit"] == "both" else None
        s["post_rstd"] = torch.zeros(rows, device="cuda") if c["post"] else None
        s["pre_rstd"] = torch.zeros(rows, device="cuda")
        return s
    # what the forward left: r and the norms' factors
    s["r"] = _values(g, rows, cols, "x", dt, pad)
    s["pre_rstd"] = _rstd(s["r"][:, :cols].float())
    s["post_rstd"] = _rstd(s["y"][:, :cols].float()) if c["post"] else None
    s["dr"] = _values(g, rows, cols, "dy", dt, pad)
    s["dh"] = _values(g, rows, cols, "dy", dt, pad)
    s["dx"] = torch.zeros((rows, cols + pad), dtype=TDT[dt], device="cuda")
    s["dy"] = torch.zeros((rows, cols + pad), dtype=TDT[dt], device="cuda")
    s["dpre_w"] = torch.zeros(cols, device="cuda")
    s["dpost_w"] = torch.zeros(cols, device="cuda") if c["post"] else None
    s["dgate"] = torch.zeros((groups, cols), device="cuda") if groups else None
    chunks = groups * ((c["gate_rows"] + 15) // 16) if groups else (rows + 15) // 16
    s["workspace"] = torch.zeros(2 * chunks * cols, device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms (32 bits, elementary operations)
def _pow2(e):
    """2^e, exactly, of int32 exponents in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x, fmt, block_rows):
    """(FP8 codes, exponent bytes) of fp32 x: of a block with a = max |x|, byte 127 - e, e = floor(log2(fmax / a))."""
    rows, cols = x.shape
    nr, nc = (rows + block_rows - 1) // block_rows, (cols + BLOCK - 1) // BLOCK
    p = x
    if rows != nr * block_rows or cols != nc * BLOCK:
        p = torch.zeros((nr * block_rows, nc * BLOCK), dtype=torch.float32, device=x.device)
        p[:rows, :cols] = x
    p = p.reshape(nr, block_rows, nc, BLOCK)
    a = p.abs().amax((1, 3))
    mant, e = torch.frexp(a)
    up = FEMAX[fmt] - (e - 1) - (2 * mant > 1.75).to(torch.int32)  # fmax = 1.75 * 2^emax
    up = torch.where(a == 0, torch.full_like(up, 126), up.clamp(-126, 126))
    q = (p * _pow2(up)[:, None, :, None]).to(TORCH_FP8[fmt]).view(torch.uint8).reshape(nr * block_rows, nc * BLOCK)
    return q[:rows, :cols].contiguous().view(TORCH_FP8[fmt]), (127 - up).to(torch.uint8)


def _decode(o):
    """The fp32 values of an operand's codes."""
    step = _pow2(o["exps"][:, :_blocks(o["cols"])[0]].to(torch.int32) - 127)
    step = step.repeat_interleave(BLOCK, 1)[:, :o["cols"]].repeat_interleave(o["block_rows"], 0)[:o["rows"]]
    return o["q"][:, :o["cols"]].contiguous().view(TORCH_FP8[o["fmt"]]).float() * step


def _coded(codes, exps):
    """Codes and scales as the values they stand for."""
    return {"codes": codes, "scales": exps.contiguous().view(torch.float8_e8m0fnu)}


def _plain_cast(s):
    c = s["case"]
    x = s["x"][:, :c["cols"]].float()
    out = {"row": _coded(*_encode(x, c["fmt"], c["block_rows"]))}
    if c["transposed"]:
        out["col"] = _coded(*_encode(x.t().contiguous(), c["fmt"], c["block_rows"]))
    return out


def _plain_product(s):
    c = s["case"]
    d = torch.matmul(_decode(s["a"]), _decode(s["b"]).t())
    if c["residual"] and c["kind"] == "wgrad":
        d = d + s["d"][:, :c["n"]].float()
        s["d"][:, :c["n"]] = d.to(TDT[c["out"]])
        return {"d": s["d"][:, :c["n"]]}
    if c["residual"]:
        d = d + s["residual"][:, :c["n"]].float()
    return {"d": d.to(TDT[c["out"]])}


def _rstd(v):
    return 1.0 / torch.sqrt((v * v).mean(1) + EPS)


def _gates(s):
    c = s["case"]
    if s["gate"] is None:
        return 1.0
    return s["gate"].float().repeat_interleave(c["gate_rows"], 0)[:c["rows"]]


def _plain_norm(s):
    c = s["case"]
    cols, dt = c["cols"], TDT[c["dtype"]]
    p, out = s["y"][:, :cols].float(), {}
    if c["post"]:
        out["post_rstd"] = _rstd(p)
        p = p * out["post_rstd"][:, None] * (s["post_w"].float() + c["offset"])
    r = (c["xs"] * s["x"][:, :cols].float() + c["ys"] * _gates(s) * p).to(dt)
    out["r"] = r
    r = r.float()  # the second norm is of the stream as it is kept
    out["pre_rstd"] = _rstd(r)
    h = r * out["pre_rstd"][:, None] * (s["pre_w"].float() + c["offset"])
    if c["emit"] == "dense":
        out["h"] = h.to(dt)
    else:
        out["row"] = _coded(*_encode(h, "e4m3", 1))
    if c["emit"] == "both":
        out["col"] = _coded(*_encode(h.t().contiguous(), "e4m3", 1))
    return out


def _plain_grad(s):
    c = s["case"]
    cols, dt = c["cols"], TDT[c["dtype"]]
    r, y = s["r"][:, :cols].float(), s["y"][:, :cols].float()
    dr, dh = s["dr"][:, :cols].float(), s["dh"][:, :cols].float()
    rn = r * s["pre_rstd"][:, None]
    out = {"dpre_w": (dh * rn).sum(0)}
    dn = dh * (s["pre_w"].float() + c["offset"])
    dr = dr + s["pre_rstd"][:, None] * (dn - rn * (dn * rn).mean(1, keepdim=True))
    out["dx"] = (c["xs"] * dr).to(dt)
    yn = y * s["post_rstd"][:, None] if c["post"] else y
    w = s["post_w"].float() + c["offset"] if c["post"] else 1.0
    db = c["ys"] * dr  # of gate * p
    if s["gate"] is not None:
        groups = s["gate"].shape[0]
        each = torch.zeros((groups * c["gate_rows"], cols), device=r.device)
        each[:c["rows"]] = db * yn * w
        out["dgate"] = each.reshape(groups, c["gate_rows"], cols).sum(1)
    dp = db * _gates(s)
    if c["post"]:
        out["dpost_w"] = (dp * yn).sum(0)
        dp = dp * w
        dp = s["post_rstd"][:, None] * (dp - yn * (dp * yn).mean(1, keepdim=True))
    out["dy"] = dp.to(dt)
    return out


# ------------------------------------------------------------------ the framework's operators
def _ok(status):
    if status != "OK":
        raise RuntimeError(status)


def _blocked(qe, o):
    if o is None:
        return None
    return qe.make_blocked(o["q"], o["q"].shape[1], o["exps"], o["exps"].shape[1], qe.E4M3 if o["fmt"] == "e4m3" else qe.E5M2,
                           o["block_rows"])


def _matrix(qe, t):
    return None if t is None else qe.make_matrix(t, t.shape[1], qe.BF16 if t.dtype == torch.bfloat16 else qe.F32)


def _own_coded(o):
    return _coded(o["q"][:, :o["cols"]].view(TORCH_FP8[o["fmt"]]), o["exps"][:, :_blocks(o["cols"])[0]])


def _own_cast(qe, s):
    c, x = s["case"], s["x"]
    _ok(qe.qe_quantize_fp8_block(_matrix(qe, x), c["rows"], c["cols"], _blocked(qe, s["row"]), _blocked(qe, s["col"])))
    return {k: _own_coded(s[k]) for k in ("row", "col") if s[k] is not None}


def _own_product(qe, s):
    c, d = s["case"], s["d"]
    dt = qe.BF16 if c["out"] == "bf16" else qe.F32
    r = s["residual"] if s["residual"] is not None else (d if c["residual"] else None)
    epi = None if r is None else qe.make_epilogue(residual=r, residual_dtype=qe.BF16 if r.dtype == torch.bfloat16 else qe.F32,
                                                  ld_residual=r.shape[1])
    _ok(qe.qe_fp8_gemm_block(_blocked(qe, s["a"]), _blocked(qe, s["b"]), c["m"], c["n"], c["k"], epi, d, dt, d.shape[1]))
    return {"d": d[:, :c["n"]]}


def _residual(qe, s):
    c = s["case"]
    dt = qe.BF16 if c["dtype"] == "bf16" else qe.F32
    return qe.make_residual(x_scale=c["xs"], y_scale=c["ys"], post_norm=c["post"], post_weight=s["post_w"], post_eps=EPS,
                            pre_norm=True, pre_weight=s["pre_w"], pre_eps=EPS, weight_dtype=dt, weight_offset=c["offset"],
                            gate=s["gate"], gate_dtype=dt, ld_gate=c["cols"], gate_rows=c["gate_rows"])


def _own_norm(qe, s):
    c = s["case"]
    _ok(qe.qe_residual_norm(_matrix(qe, s["x"]), _matrix(qe, s["y"]), c["rows"], c["cols"], _residual(qe, s), _matrix(qe, s["r"]),
                            _matrix(qe, s["h"]), _blocked(qe, s["row"]), _blocked(qe, s["col"]), s["post_rstd"], s["pre_rstd"]))
    out = {k: s[k][:, :c["cols"]] for k in ("r", "h") if s[k] is not None}
    out.update({k: _own_coded(s[k]) for k in ("row", "col") if s[k] is not None})
    out.update({k: s[k] for k in ("post_rstd", "pre_rstd") if s[k] is not None})
    return out


def _own_grad(qe, s):
    c = s["case"]
    _ok(qe.qe_residual_norm_grad(_matrix(qe, s["dr"]), _matrix(qe, s["dh"]), _matrix(qe, s["r"]), _matrix(qe, s["y"]), c["rows"],
                                 c["cols"], _residual(qe, s), s["post_rstd"], s["pre_rstd"], _matrix(qe, s["dx"]),
                                 _matrix(qe, s["dy"]), s["dpost_w"], s["dpre_w"], s["dgate"], qe.INIT, s["workspace"]))
    out = {k: s[k][:, :c["cols"]] for k in ("dx", "dy")}
    out.update({k: s[k] for k in ("dpre_w", "dpost_w", "dgate") if s[k] is not None})
    return out


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"cast": _plain_cast, "product": _plain_product, "norm": _plain_norm, "grad": _plain_grad}[op](state)
    from paper_2609_23536_amd import qe
    return {"cast": _own_cast, "product": _own_product, "norm": _own_norm, "grad": _own_grad}[op](qe, state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    code = 1 + 1 / BLOCK  # a code and its share of a scale
    if c["op"] == "product":
        m, n, k, e = c["m"], c["n"], c["k"], ESIZE[c["out"]]
        b = m * k * code + n * k * (code if c["kind"] == "wgrad" else 1) + m * n * e + (m * n * e if c["residual"] else 0)
        return {"bytes": b, "flops": 2 * m * n * k}
    v, e = c["rows"] * c["cols"], ESIZE[c["dtype"]]
    if c["op"] == "cast":
        return {"bytes": v * (e + (code if c["block_rows"] == 1 else 1) * (2 if c["transposed"] else 1)), "flops": 0}
    gates = 0 if not c["gate_rows"] else (c["rows"] + c["gate_rows"] - 1) // c["gate_rows"] * c["cols"]
    if c["op"] == "norm":
        return {"bytes": v * (3 * e + {"dense": e, "row": code, "both": 2 * code}[c["emit"]]) + gates * e, "flops": 0}
    return {"bytes": v * 6 * e + gates * (e + 4), "flops": 0}


# ------------------------------------------------------------------ the same in 64 bits
def _step(n):
    """2^n in 64 bits, of whole numbers n: by its bits, as powers are not exact on every device."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_codes(x, fmt, br):
    """(codes, scales), in 64 bits, of float64 x."""
    rows, cols = x.shape
    f = torch.nn.functional.pad(x, (0, -cols % BLOCK, 0, -rows % br))
    shape = (f.shape[0] // br, br, f.shape[1] // BLOCK, BLOCK)
    f = f.reshape(shape)
    amax = f.abs().amax(3).amax(1).clamp(min=2.0 ** -140)
    step = _step(-torch.floor(torch.log2(FMAX[fmt] / amax)).clamp(max=126))
    v = (f / step[:, None, :, None]).reshape(shape[0] * br, -1)[:rows, :cols]
    # round to the format's grid: 3 or 2 fraction bits, exponents from -6 or -14 up
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = torch.frexp(v)
    grid = _step((e - 1).clamp(min=low) - bits)
    return {"codes": torch.round(v / grid) * grid, "scales": step}


def _exact_values(o):
    step = _step(o["exps"].to(torch.int64) - 127)
    at_r = torch.arange(o["rows"], device="cuda") // o["block_rows"]
    at_c = torch.arange(o["cols"], device="cuda") // BLOCK
    return o["q"][:, :o["cols"]].contiguous().view(TORCH_FP8[o["fmt"]]).double() * step[at_r][:, at_c]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "product":
        d = _exact_values(s["a"]) @ _exact_values(s["b"]).t()
        if c["residual"]:
            d += (s["d"] if s["residual"] is None else s["residual"])[:, :c["n"]].double()
        return {"d": d}
    cols, rows = c["cols"], c["rows"]
    if c["op"] == "cast":
        x = s["x"][:, :cols].double()
        out = {"row": _exact_codes(x, c["fmt"], c["block_rows"])}
        if c["transposed"]:
            out["col"] = _exact_codes(x.t().contiguous(), c["fmt"], c["block_rows"])
        return out
    w = {k: (s[k].double() + c["offset"] if s[k] is not None else None) for k in ("pre_w", "post_w")}
    gate = torch.ones((1, 1), dtype=torch.float64, device="cuda")
    at = torch.zeros(rows, dtype=torch.int64, device="cuda")
    if s["gate"] is not None:
        gate, at = s["gate"].double(), torch.arange(rows, device="cuda") // c["gate_rows"]
    y = s["y"][:, :cols].double()
    inv = lambda v: (v.square().sum(1) / cols + EPS).rsqrt()  # noqa: E731
    if c["op"] == "norm":
        out = {}
        if c["post"]:
            out["post_rstd"] = inv(y)
            y = y * out["post_rstd"].unsqueeze(1) * w["post_w"]
        out["r"] = s["x"][:, :cols].double() * c["xs"] + y * gate[at] * c["ys"]
        kept = out["r"].to(TDT[c["dtype"]]).double()
        out["pre_rstd"] = inv(kept)
        h = kept * out["pre_rstd"].unsqueeze(1) * w["pre_w"]
        if c["emit"] == "dense":
            out["h"] = h
        else:
            out["row"] = _exact_codes(h, "e4m3", 1)
        if c["emit"] == "both":
            out["col"] = _exact_codes(h.t().contiguous(), "e4m3", 1)
        return out
    # Jacobians: d(v f)/dv = f (1 - (v f)(v f)^T / cols) with f = 1 / rms(v)
    def back(d, v, f):
        n = v * f
        return f * (d - n * torch.linalg.vecdot(d, n).unsqueeze(1) / cols)
    r, dh = s["r"][:, :cols].double(), s["dh"][:, :cols].double()
    fr = s["pre_rstd"].double().unsqueeze(1)
    total = s["dr"][:, :cols].double() + back(dh * w["pre_w"], r, fr)
    out = {"dpre_w": torch.linalg.vecdot(dh, r * fr, dim=0), "dx": total * c["xs"]}
    fy = s["post_rstd"].double().unsqueeze(1) if c["post"] else torch.ones((1, 1), dtype=torch.float64, device="cuda")
    p = y * fy * (w["post_w"] if c["post"] else 1.0)
    if s["gate"] is not None:
        out["dgate"] = torch.zeros((gate.shape[0], cols), dtype=torch.float64, device="cuda").index_add_(0, at, total * p * c["ys"])
    dp = total * gate[at] * c["ys"]
    if c["post"]:
        out["dpost_w"] = torch.linalg.vecdot(dp, y * fy, dim=0)
        dp = back(dp * w["post_w"], y, fy)
    out["dy"] = dp
    return out
