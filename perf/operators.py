"""The operators between a stage's FP8 linears, as a training or serving program calls them, and their plain forms.

Four kinds of case:

* ``product``: an FP8 product with bias, activation and residual in its epilogue.  With ``train`` the forward also
  saves its pre-activation and the gradient through the activation is taken from it: one training pass.
* ``gated``: the two projections of a gated feed-forward, its activation and product; ``train`` as above.
* ``grad``: the gradient through an activation (or a gated pair) from what the forward saved, emitted as the FP8 codes
  that the dI and dW products read, with the amax, the scale update and the bias gradient.
* ``checkpoint``: an activation stored in 8 bits in the forward and restored in the backward.

Inputs are seeded and made on the GPU: X ~ N(0, 1), W ~ N(0, 0.02), gradients ~ N(0, 0.01), residuals ~ N(0, 1).
"""
import math

import torch

own = False

FMAX = {"e4m3": 448.0, "e5m2": 57344.0}
FEMAX = {"e4m3": 8, "e5m2": 15}
TORCH_FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"none": 0, "f32": 4, "bf16": 2, "i8": 33 / 32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
GROUP = 32          # columns of a row that share one exponent in an 8-bit checkpoint
AMAX_FLOATS = 4096  # an amax accumulator
HISTORY = 16


def _product(**kw):
    case = {"op": "product", "m": 1, "n": 1, "k": 1, "fmt_a": "e4m3", "fmt_b": "e4m3", "bias": "none", "act": "none",
            "residual": "none", "out": "bf16", "saved": "none", "train": False, "pad": 0}
    case.update(kw)
    return case


def _gated(**kw):
    case = {"op": "gated", "m": 1, "n": 1, "k": 1, "fmt_a": "e4m3", "fmt_b": "e4m3", "act": "silu", "out": "bf16",
            "saved": "none", "train": False, "pad": 0}
    case.update(kw)
    return case


def _grad(**kw):
    case = {"op": "grad", "rows": 1, "cols": 1, "gated": False, "act": "silu", "saved": "i8", "dtype": "bf16",
            "fmt": "e5m2", "dense": "none", "bias": False, "pad": 0}
    case.update(kw)
    return case


def listed():
    return [
        # The down projection of one token being served, added to the residual stream.
        _product(name="product_1x4096x14336", m=1, n=4096, k=14336, residual="bf16"),
        # Ragged sizes (nothing a multiple of 16), odd row strides, every part of the epilogue, E5M2 by E4M3.
        _product(name="product_1000x2730x1365", m=1000, n=2730, k=1365, fmt_a="e5m2", bias="f32", act="gelu",
                 residual="bf16", pad=3),
        # A biased layer of the single-linear workload in a training pass, pre-activations kept in 16 bits.
        _product(name="product_train_128x256x256", m=128, n=256, k=256, bias="bf16", act="gelu_tanh", saved="bf16",
                 train=True),
        # The down projection of the Llama-3-70B-shaped stage with its residual.
        _product(name="product_8192x8192x28672", m=8192, n=8192, k=28672, residual="bf16"),
        # The gated feed-forward of one token being served (Llama-3-8B-shaped).
        _gated(name="gated_1x14336x4096", m=1, n=14336, k=4096),
        # A ragged batch of prompt tokens.
        _gated(name="gated_333x2730x1365", m=333, n=2730, k=1365, act="gelu_tanh", pad=3),
        # A microbatch of the Llama-3-8B-shaped stage in training: forward with 8-bit checkpoints, gradient from them.
        _gated(name="gated_train_4096x14336x4096", m=4096, n=14336, k=4096, saved="i8", train=True),
        # The gradient of the largest gated pair of the Llama-3-70B-shaped stage, straight to codes.
        _grad(name="grad_gated_8192x28672", rows=8192, cols=28672, gated=True),
        # A ragged biased layer, fp32 gradients, with the dense gradient as well.
        _grad(name="grad_bias_1000x2730_f32", rows=1000, cols=2730, act="gelu", dtype="f32", dense="f32", bias=True,
              pad=3),
        # A zero-bubble microbatch of the Llama-3-8B-shaped stage.
        _grad(name="grad_gated_2048x14336", rows=2048, cols=14336, gated=True),
        # The input of the Llama-3-8B-shaped stage, kept in 8 bits.
        {"op": "checkpoint", "name": "checkpoint_4096x14336", "rows": 4096, "cols": 14336, "dtype": "bf16",
         "out": "bf16", "pad": 0},
        # Odd rows, fp32.
        {"op": "checkpoint", "name": "checkpoint_1500x4099_f32", "rows": 1500, "cols": 4099, "dtype": "f32",
         "out": "bf16", "pad": 3},
    ]


def _log_int(rng, lo, hi, odd=0.4):
    """A size spread over the logarithm of [lo, hi]: any integer, or (more often) a multiple of 64 where that fits."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() >= odd and v >= 96:
        v = (v + 32) // 64 * 64
    v = max(lo, min(hi, v))
    return v - 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(("product", "product", "gated", "gated", "grad", "grad", "checkpoint"))
    if op in ("product", "gated"):
        while True:
            m = rng.choice((1, rng.randint(2, 16), _log_int(rng, 17, 8192), _log_int(rng, 17, 8192)))
            n, k = _log_int(rng, 32, 28672), _log_int(rng, 64, 28672)
            if (2.0 if op == "product" else 4.0) * m * n * k <= 3.8e12 and n * k <= 28672 * 8192:
                break
        train = m > 16 and rng.random() < 0.5
        saved = rng.choice(("i8", "i8", "bf16")) if train else "none"
        fmts = {"fmt_a": rng.choice(("e4m3", "e4m3", "e5m2")), "fmt_b": rng.choice(("e4m3", "e4m3", "e5m2"))}
        common = {"m": m, "n": n, "k": k, "saved": saved, "train": train, "out": "bf16",
                  "pad": rng.choice((0, 0, 3, 16)), **fmts}
        # relu's slope jumps at a pre-activation of zero, so a training pass through it has no value to compare with there
        acts = [a for a in ACTS if not (train and a == "relu")]
        if op == "gated":
            return _gated(act=rng.choice(("silu", "silu", *acts)), **common)
        return _product(bias=rng.choice(("none", "bf16", "f32")), act=rng.choice(acts),
                        residual=rng.choice(("none", "bf16", "bf16", "f32")), **common)
    while True:
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 32, 28672)
        if rows * cols <= 8192 * 28672 and rows * cols >= 4096:
            break
    if op == "checkpoint":
        return {"op": "checkpoint", "rows": rows, "cols": cols, "dtype": rng.choice(("bf16", "bf16", "f32")),
                "out": rng.choice(("bf16", "bf16", "f32")), "pad": rng.choice((0, 0, 3, 16))}
    gated = rng.random() < 0.6
    return _grad(rows=rows, cols=cols, gated=gated, act=rng.choice(ACTS if gated else ACTS[1:]),
                 saved=rng.choice(("i8", "i8", "bf16")), dtype=rng.choice(("bf16", "bf16", "f32")),
                 fmt=rng.choice(("e5m2", "e5m2", "e4m3")), dense=rng.choice(("none", "none", "bf16", "f32")),
                 bias=not gated and rng.random() < 0.5, pad=rng.choice((0, 0, 3, 16)))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, rows, cols, sigma, dtype, pad=0):
    """[rows, cols] values in rows of cols + pad."""
    x = torch.zeros((rows, cols + pad), dtype=TDT[dtype], device="cuda")
    chunk = max(1, (1 << 27) // cols)  # rows at a time, drawn in fp32 and rounded
    for r in range(0, rows, chunk):
        n = min(chunk, rows - r)
        x[r:r + n, :cols] = torch.randn((n, cols), generator=g, device="cuda") * sigma
    return x


def _up16(v):
    return (v + 15) // 16 * 16


def _exponent(amax, fmt):
    """floor(log2(fmax / amax)): fmax = 1.75 * 2^emax, amax = (2 m) * 2^(e - 1)."""
    m, e = math.frexp(amax)
    return max(-126, min(126, FEMAX[fmt] - (e - 1) - (1 if 2 * m > 1.75 else 0)))


def _codes(g, rows, k, fmt, sigma):
    """FP8 codes of normal values at the scale of their amax, row stride a multiple of 16, and the scale's inverse."""
    q = torch.zeros((rows, _up16(k)), dtype=torch.uint8, device="cuda")
    x = _normal(g, rows, k, sigma, "f32")
    e = _exponent(float(x.abs().max()), fmt)
    q[:, :k] = (x * 2.0 ** e).clamp(-FMAX[fmt], FMAX[fmt]).to(TORCH_FP8[fmt]).view(torch.uint8)
    return q, torch.tensor([2.0 ** -e], dtype=torch.float32, device="cuda")


def _saved_buffers(rows, cols, kind):
    """What a program keeps for the backward: bf16 values, or codes and exponents."""
    if kind == "none":
        return None
    data = torch.zeros((rows, cols), dtype=torch.bfloat16 if kind == "bf16" else torch.int8, device="cuda")
    exps = torch.zeros((rows, (cols + GROUP - 1) // GROUP), dtype=torch.uint8, device="cuda") if kind == "i8" else None
    return {"kind": kind, "data": data, "exps": exps}


def _outs(*shape, kind):
    return None if kind == "none" else torch.zeros(shape, dtype=TDT[kind], device="cuda")


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"case": c}
    if c["op"] in ("product", "gated"):
        m, n, k = c["m"], c["n"], c["k"]
        s["a"], s["a_inv"] = _codes(g, m, k, c["fmt_a"], 1.0)
        s["b"], s["b_inv"] = _codes(g, n * (2 if c["op"] == "gated" else 1), k, c["fmt_b"], 0.02)
        s["d"] = torch.zeros((m, n + c["pad"]), dtype=TDT[c["out"]], device="cuda")
        if c["op"] == "product":
            s["bias"] = None if c["bias"] == "none" else _normal(g, 1, n, 0.5, c["bias"]).reshape(-1)
            s["residual"] = None if c["residual"] == "none" else _normal(g, m, n, 1.0, c["residual"], c["pad"])
        pair = 2 if c["op"] == "gated" else 1
        s["saved"] = [_saved_buffers(m, n, c["saved"]) for _ in range(pair)]
        if c["train"]:
            s["dd"] = _normal(g, m, n, 0.01, "bf16")
            s["dz"] = torch.zeros((m, n * pair), dtype=torch.bfloat16, device="cuda")
        return s
    rows, cols, pad = c["rows"], c["cols"], c["pad"]
    if c["op"] == "checkpoint":
        s["x"] = _normal(g, rows, cols, 1.0, c["dtype"], pad)
        s["saved"] = [_saved_buffers(rows, cols, "i8")]
        s["restored"] = torch.zeros((rows, cols), dtype=TDT[c["out"]], device="cuda")
        return s
    pair = 2 if c["gated"] else 1
    width = cols * pair
    s["dd"] = _normal(g, rows, cols, 0.01, c["dtype"], pad)
    s["saved"] = []
    for _ in range(pair):
        v, x = _saved_buffers(rows, cols, c["saved"]), _normal(g, rows, cols, 1.28, "f32")
        if c["saved"] == "bf16":
            v["data"].copy_(x)
        else:
            v["data"], v["exps"] = _pack(x)
        s["saved"].append(v)
    s["dz"] = _outs(rows, width + pad, kind=c["dense"])
    s["dbias"] = torch.zeros(width, dtype=torch.float32, device="cuda") if c["bias"] else None
    s["workspace"] = torch.zeros(((rows + 63) // 64) * width, dtype=torch.float32, device="cuda") if c["bias"] else None
    s["q_row"] = torch.zeros((rows, _up16(width)), dtype=torch.uint8, device="cuda")
    s["q_col"] = torch.zeros((width, _up16(rows)), dtype=torch.uint8, device="cuda")
    s["hist"] = torch.zeros(HISTORY, dtype=torch.float32, device="cuda")
    e = _exponent(0.16, c["fmt"])  # the step before had gradients of this size
    s["scale"] = torch.tensor([2.0 ** e], dtype=torch.float32, device="cuda")
    s["inv"] = torch.tensor([2.0 ** -e], dtype=torch.float32, device="cuda")
    s["snapshot"] = torch.zeros(1, dtype=torch.float32, device="cuda")
    s["accum"] = torch.zeros(AMAX_FLOATS, dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms (32 bits, elementary operations)
def _decode(q, k, fmt):
    return q[:, :k].contiguous().view(TORCH_FP8[fmt]).float()


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        a = math.sqrt(2.0 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _pow2(e):
    """2^e, exactly, of int32 exponents in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pack(x):
    """(codes, exponents) of the 8-bit checkpoint of fp32 x."""
    rows, cols = x.shape
    groups = (cols + GROUP - 1) // GROUP
    p = torch.zeros((rows, groups * GROUP), dtype=torch.float32, device=x.device)
    p[:, :cols] = x
    p = p.reshape(rows, groups, GROUP)
    mant, e = torch.frexp(p.abs().amax(2))
    s = 6 - (e - 1) - (2 * mant > 127.0 / 64.0).to(torch.int32)  # 127 = (127 / 64) * 2^6
    s = torch.where(mant == 0, torch.full_like(s, 126), s.clamp(-126, 126))
    q = torch.round(p * _pow2(s).unsqueeze(2)).to(torch.int8).reshape(rows, groups * GROUP)[:, :cols].contiguous()
    return q, (127 - s).to(torch.uint8)


def _unpack(q, exps):
    cols = q.shape[1]
    step = _pow2(exps.to(torch.int32) - 127)
    return q.float() * step.repeat_interleave(GROUP, 1)[:, :cols]


def _kept(z, kind):
    """z as the backward pass finds it."""
    return _unpack(*_pack(z)) if kind == "i8" else z.to(torch.bfloat16).float()


def _slopes(dd, zs, act):
    """The gradient of act(z) (one saved tensor) or of act(g) * u (two), side by side."""
    if len(zs) == 1:
        return dd * _act_slope(zs[0], act)
    return torch.cat((dd * zs[1] * _act_slope(zs[0], act), dd * _act(zs[0], act)), 1)


def _plain_product(s):
    c = s["case"]
    m, n, k = c["m"], c["n"], c["k"]
    z = torch.matmul(_decode(s["a"], k, c["fmt_a"]), _decode(s["b"], k, c["fmt_b"]).t()) * (s["a_inv"] * s["b_inv"])
    if c["op"] == "gated":
        zs = [z[:, :n], z[:, n:]]
        d = _act(zs[0], c["act"]) * zs[1]
    else:
        z = z if s["bias"] is None else z + s["bias"].float()
        zs, d = [z], _act(z, c["act"])
        d = d if s["residual"] is None else d + s["residual"][:, :n].float()
    out = {"d": d.to(TDT[c["out"]])}
    if c["train"]:
        out["dz"] = _slopes(s["dd"].float(), [_kept(t, c["saved"]) for t in zs], c["act"]).to(torch.bfloat16)
    return out


def _plain_grad(s):
    c = s["case"]
    zs = [v["data"].float() if c["saved"] == "bf16" else _unpack(v["data"], v["exps"]) for v in s["saved"]]
    dz = _slopes(s["dd"][:, :c["cols"]].float(), zs, c["act"])
    f = FMAX[c["fmt"]]
    q = (dz * s["scale"]).clamp(-f, f).to(TORCH_FP8[c["fmt"]])
    out = {"q_row": q, "q_col": q.view(torch.uint8).t().contiguous().view(TORCH_FP8[c["fmt"]]), "snapshot": s["inv"].clone()}
    if c["dense"] != "none":
        out["dz"] = dz.to(TDT[c["dense"]])
    if c["bias"]:
        out["dbias"] = dz.sum(0)
    # the scale update: this step's amax enters the history, the scale follows the largest
    hist = s["hist"]
    hist[0] = torch.maximum(hist[0], dz.abs().max())
    mant, e = torch.frexp(hist.max())
    up = FEMAX[c["fmt"]] - (e - 1) - (2 * mant > 1.75).to(torch.int32)
    s["scale"].copy_(_pow2(up))
    s["inv"].copy_(_pow2(-up))
    s["hist"] = torch.cat((torch.zeros_like(hist[:1]), hist[2:], hist[:1]))
    out.update(hist=s["hist"], scale=s["scale"])
    return out


def _plain_checkpoint(s):
    c = s["case"]
    return {"restored": _unpack(*_pack(s["x"][:, :c["cols"]].float())).to(TDT[c["out"]])}


# ------------------------------------------------------------------ the framework's operators
def _ok(status):
    if status != "OK":
        raise RuntimeError(status)


def _consts(qe):
    return ({"e4m3": qe.E4M3, "e5m2": qe.E5M2}, {"f32": qe.F32, "bf16": qe.BF16, "none": qe.F32},
            {"none": qe.ACT_NONE, "relu": qe.ACT_RELU, "gelu": qe.ACT_GELU, "gelu_tanh": qe.ACT_GELU_TANH,
             "silu": qe.ACT_SILU})


def _handle(qe, v):
    if v is None:
        return None
    if v["kind"] == "bf16":
        return qe.make_saved(qe.SAVED_BF16, v["data"], v["data"].shape[1])
    return qe.make_saved(qe.SAVED_I8, v["data"], v["data"].shape[1], v["exps"], v["exps"].shape[1])


def _own_product(qe, s):
    c = s["case"]
    fmt, dt, act = _consts(qe)
    m, n, k, d, a, b = c["m"], c["n"], c["k"], s["d"], s["a"], s["b"]
    saved = [_handle(qe, v) for v in s["saved"]]
    if c["op"] == "gated":
        _ok(qe.qe_fp8_gemm_gated(a, fmt[c["fmt_a"]], a.shape[1], b, b[n:], fmt[c["fmt_b"]], b.shape[1], m, n, k,
                                 s["a_inv"], s["b_inv"], s["b_inv"], act[c["act"]], d, dt[c["out"]], d.shape[1],
                                 saved[0], saved[1]))
    else:
        r = s["residual"]
        epi = qe.make_epilogue(act[c["act"]], s["bias"], dt[c["bias"]], r, dt[c["residual"]],
                               0 if r is None else r.shape[1], saved[0])
        _ok(qe.qe_fp8_gemm_act(a, fmt[c["fmt_a"]], a.shape[1], b, fmt[c["fmt_b"]], b.shape[1], m, n, k, s["a_inv"],
                               s["b_inv"], epi, d, dt[c["out"]], d.shape[1]))
    out = {"d": d[:, :n]}
    if c["train"]:
        dz = s["dz"]
        _ok(qe.qe_act_grad(s["dd"], qe.BF16, n, m, n, act[c["act"]], saved[0], saved[1] if c["op"] == "gated" else None,
                           dz=dz, dz_dtype=qe.BF16, ld_dz=dz.shape[1]))
        out["dz"] = dz
    return out


def _own_grad(qe, s):
    c = s["case"]
    fmt, dt, act = _consts(qe)
    rows, cols, dd, dz, qr, qc = c["rows"], c["cols"], s["dd"], s["dz"], s["q_row"], s["q_col"]
    width = cols * (2 if c["gated"] else 1)
    meta = qe.make_meta(s["hist"], s["scale"], s["inv"], fmt[c["fmt"]], 0, s["accum"])
    saved = [_handle(qe, v) for v in s["saved"]]
    _ok(qe.qe_act_grad(dd, dt[c["dtype"]], dd.shape[1], rows, cols, act[c["act"]], saved[0],
                       saved[1] if c["gated"] else None, meta=meta, q_row=qr, ld_row=qr.shape[1], q_col=qc,
                       ld_col=qc.shape[1], scale_inv_snapshot=s["snapshot"], dz=dz, dz_dtype=dt[c["dense"]],
                       ld_dz=0 if dz is None else dz.shape[1], dbias=s["dbias"], workspace=s["workspace"]))
    _ok(qe.qe_amax_scale_update([meta]))
    f8 = TORCH_FP8[c["fmt"]]
    out = {"q_row": qr[:, :width].view(f8), "q_col": qc[:, :rows].view(f8), "snapshot": s["snapshot"],
           "hist": s["hist"], "scale": s["scale"]}
    if dz is not None:
        out["dz"] = dz[:, :width]
    if c["bias"]:
        out["dbias"] = s["dbias"]
    return out


def _own_checkpoint(qe, s):
    c = s["case"]
    _, dt, _ = _consts(qe)
    x, saved = s["x"], _handle(qe, s["saved"][0])
    _ok(qe.qe_act_save(x, dt[c["dtype"]], x.shape[1], c["rows"], c["cols"], saved))
    _ok(qe.qe_act_restore(saved, c["rows"], c["cols"], s["restored"], dt[c["out"]], c["cols"]))
    return {"restored": s["restored"]}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"product": _plain_product, "gated": _plain_product, "grad": _plain_grad,
                "checkpoint": _plain_checkpoint}[op](state)
    from paper_2609_23536_amd import qe
    return {"product": _own_product, "gated": _own_product, "grad": _own_grad, "checkpoint": _own_checkpoint}[op](qe, state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] in ("product", "gated"):
        m, n, k, pair = c["m"], c["n"], c["k"], 2 if c["op"] == "gated" else 1
        b = m * k + pair * n * k + m * n * ESIZE[c["out"]] + pair * m * n * ESIZE[c["saved"]]
        if c["op"] == "product":
            b += n * ESIZE[c["bias"]] + m * n * ESIZE[c["residual"]]
        if c["train"]:  # the saved values and the gradient in, dz out
            b += pair * m * n * (ESIZE[c["saved"]] + 2) + m * n * 2
        return {"bytes": b, "flops": 2 * m * n * k * pair}
    e = c["rows"] * c["cols"]
    if c["op"] == "checkpoint":
        return {"bytes": e * (ESIZE[c["dtype"]] + 2 * ESIZE["i8"] + ESIZE[c["out"]]), "flops": 0}
    pair = 2 if c["gated"] else 1
    return {"bytes": e * (ESIZE[c["dtype"]] + pair * (ESIZE[c["saved"]] + 2 + ESIZE[c["dense"]])) + 8 * HISTORY,
            "flops": 0}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_act(z, act):
    """(value, derivative)."""
    if act == "relu":
        return z.relu(), torch.heaviside(z, torch.zeros_like(z))
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":  # (1 + tanh v) / 2 = sigmoid(2 v)
        a = 2 * math.sqrt(2 / math.pi)
        p = torch.sigmoid(a * (z + 0.044715 * z ** 3))
        return z * p, p + z * p * (1 - p) * a * (1 + 0.134145 * z.square())
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    return z, torch.ones_like(z)


def _exact_kept(x, kind):
    if kind == "bf16":
        return x.float().to(torch.bfloat16).double()
    rows, cols = x.shape
    full = torch.nn.functional.pad(x, (0, -cols % GROUP)).reshape(rows, -1, GROUP)
    amax = full.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -120)
    step = torch.exp2(-torch.floor(torch.log2(127.0 / amax)).clamp(max=126))
    return (torch.round(full / step) * step).reshape(rows, -1)[:, :cols]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "checkpoint":
        return {"restored": _exact_kept(s["x"][:, :c["cols"]].double(), "i8")}
    if c["op"] in ("product", "gated"):
        n, k = c["n"], c["k"]
        a = s["a"][:, :k].contiguous().view(TORCH_FP8[c["fmt_a"]]).double() * s["a_inv"].double()
        b = s["b"][:, :k].contiguous().view(TORCH_FP8[c["fmt_b"]]).double() * s["b_inv"].double()
        zs = [a @ w.t() for w in b.split(n)]
        if c["op"] == "gated":
            d = _exact_act(zs[0], c["act"])[0] * zs[1]
        else:
            if s["bias"] is not None:
                zs[0] += s["bias"].double()
            d = _exact_act(zs[0], c["act"])[0]
            if s["residual"] is not None:
                d = d + s["residual"][:, :n].double()
        out = {"d": d}
        if c["train"]:
            zs = [_exact_kept(z, c["saved"]) for z in zs]
            dd, (v, slope) = s["dd"].double(), _exact_act(zs[0], c["act"])
            out["dz"] = dd * slope if len(zs) == 1 else torch.cat((dd * zs[1] * slope, dd * v), 1)
        return out
    cols, zs = c["cols"], []
    for v in s["saved"]:
        if c["saved"] == "bf16":
            zs.append(v["data"].double())
        else:
            step = torch.pow(2.0, v["exps"].double() - 127)
            at = torch.arange(cols, device="cuda") // GROUP
            zs.append(v["data"].double() * step[:, at])
    dd, (v, slope) = s["dd"][:, :cols].double(), _exact_act(zs[0], c["act"])
    dz = dd * slope if len(zs) == 1 else torch.cat((dd * zs[1] * slope, dd * v), 1)
    f = FMAX[c["fmt"]]
    q = (dz * s["scale"].double()).clamp(-f, f).float().to(TORCH_FP8[c["fmt"]]).double()
    amax = float(dz.abs().max())
    hist = torch.zeros(HISTORY, dtype=torch.float64, device="cuda")
    hist[-1] = amax
    out = {"q_row": q, "q_col": q.t().contiguous(), "snapshot": s["inv"].double(), "hist": hist,
           "scale": torch.tensor([2.0 ** _exponent(amax, c["fmt"])], dtype=torch.float64, device="cuda")}
    if c["dense"] != "none":
        out["dz"] = dz
    if c["bias"]:
        out["dbias"] = dz.sum(0)
    return out
