"""8-bit checkpoints of values near the top of the FP32 range, restored and read by the gradient, on the GPU.

A group's exponent byte is 127 - s with 2^-s its step, so groups whose largest value lies near 2^126, 2^127 and 2^128
have the bytes 247, 248 and 249.  Every value here is an integer code times its step, restored exactly; the
gradients are products with a power of two, exact too.
"""
import numpy as np
import pytest

from oracle import activation as oa
from tests.gpu_util import dev, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu
BYTES = {246: 127, 247: 127, 248: 127, 249: 63}  # byte: its largest code whose value is finite


def codes_of(byte):
    """Zeros, both signs, small and large codes, in two groups and a part of one."""
    top = BYTES[byte]
    row = np.array([top, -top, 0, 1, -1, 5, -64 if top > 64 else -17, 33] * 9, dtype=np.int8)[:70]
    return np.stack([row, -row, np.roll(row, 3)])


def on_device(byte, d):
    codes = codes_of(byte)
    exps = np.full((codes.shape[0], 3), byte, dtype=np.uint8)
    return codes, torch.from_numpy(codes).to(d), torch.from_numpy(exps).to(d)


@pytest.mark.parametrize("byte", BYTES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_restore(dtype, byte):
    qe, d = need_lib(), dev()
    codes, data, exps = on_device(byte, d)
    rows, cols = codes.shape
    t, q = {"bf16": (torch.bfloat16, qe.BF16), "f32": (torch.float32, qe.F32)}[dtype]
    x = torch.zeros((rows, cols), dtype=t, device=d)
    assert qe.qe_act_restore(qe.make_saved(qe.SAVED_I8, data, cols, exps, 3), rows, cols, x, q, cols) == "OK"
    assert np.array_equal(x.double().cpu().numpy(), codes * 2.0 ** (byte - 127))


@pytest.mark.parametrize("byte", BYTES)
def test_save_and_restore(byte):
    """The values save to the codes that they are multiples of, and come back."""
    qe, d = need_lib(), dev()
    codes, _, _ = on_device(byte, d)
    rows, cols = codes.shape
    v = codes * 2.0 ** (byte - 127)
    x = torch.from_numpy(v.astype(np.float32)).to(d)
    data, exps = torch.zeros((rows, cols), dtype=torch.int8, device=d), torch.zeros((rows, 3), dtype=torch.uint8, device=d)
    s = qe.make_saved(qe.SAVED_I8, data, cols, exps, 3)
    back = torch.zeros_like(x)
    assert qe.qe_act_save(x, qe.F32, cols, rows, cols, s) == "OK"
    assert qe.qe_act_restore(s, rows, cols, back, qe.F32, cols) == "OK"
    want = oa.pack(v)
    assert np.array_equal(data.cpu().numpy(), want[0]) and np.array_equal(exps.cpu().numpy(), want[1])
    assert np.array_equal(back.double().cpu().numpy(), oa.unpack(*want))
    assert np.array_equal(oa.unpack(*want), v)


@pytest.mark.parametrize("byte", BYTES)
@pytest.mark.parametrize("act", ["none", "relu"])
def test_gradient_of_a_gated_pair(act, byte):
    qe, d = need_lib(), dev()
    codes, data, exps = on_device(byte, d)
    rows, cols = codes.shape
    z = codes * 2.0 ** (byte - 127)
    saved = qe.make_saved(qe.SAVED_I8, data, cols, exps, 3)
    dd = torch.full((rows, cols), 2.0 ** -120, device=d)
    dz = torch.zeros((rows, 2 * cols), device=d)
    assert qe.qe_act_grad(dd, qe.F32, cols, rows, cols, {"none": qe.ACT_NONE, "relu": qe.ACT_RELU}[act], saved, saved, dz=dz,
                          dz_dtype=qe.F32, ld_dz=2 * cols) == "OK"
    assert np.array_equal(dz.double().cpu().numpy(), oa.gate_grad(np.full((rows, cols), 2.0 ** -120), z, z, act))


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_gradient_far_out(act):
    """Slopes of 1 above and of 0 below, for pre-activations whose square overflows."""
    qe, d = need_lib(), dev()
    for byte in BYTES:
        codes, data, exps = on_device(byte, d)
        rows, cols = codes.shape
        dd = torch.full((rows, cols), 0.5, device=d)
        dz = torch.zeros((rows, cols), device=d)
        a = {"gelu": qe.ACT_GELU, "gelu_tanh": qe.ACT_GELU_TANH, "silu": qe.ACT_SILU}[act]
        assert qe.qe_act_grad(dd, qe.F32, cols, rows, cols, a, qe.make_saved(qe.SAVED_I8, data, cols, exps, 3), dz=dz,
                              dz_dtype=qe.F32, ld_dz=cols) == "OK"
        want = np.where(codes > 0, 0.5, np.where(codes < 0, 0.0, 0.25))
        assert np.array_equal(dz.double().cpu().numpy(), want)


TOP = 2.0 ** 122  # the largest step
LARGEST = float(np.finfo(np.float32).max)
TOPMOST = [63.5 * TOP, np.nextafter(np.float32(63.5 * TOP), np.float32(0)), -63.5 * TOP, LARGEST, -LARGEST, 63.0 * TOP, 62.5 * TOP,
           -0.5 * TOP, 0.75 * TOP, 0.0, 255.0 * 2.0 ** 120]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [32, 45])
def test_the_largest_finite_values_stay_finite(cols, dtype):
    """Off by less than a step and never infinite; the rest of their group as ever, within half a step."""
    qe, d = need_lib(), dev()
    v = np.zeros((3, cols), dtype=np.float32)
    v[0, :len(TOPMOST)], v[1, :len(TOPMOST)], v[2, cols - 1] = TOPMOST, np.negative(TOPMOST), 255.0 * 2.0 ** 120
    t, q = {"bf16": (torch.bfloat16, qe.BF16), "f32": (torch.float32, qe.F32)}[dtype]
    if dtype == "bf16":
        v = np.where(np.abs(v) > 255.0 * 2.0 ** 120, np.sign(v) * 255.0 * 2.0 ** 120, v).astype(np.float32)
    x = torch.from_numpy(v).to(d).to(t)
    v = x.double().cpu().numpy()
    assert np.isfinite(v).all()
    groups = -(-cols // 32)
    data = torch.zeros((3, cols), dtype=torch.int8, device=d)
    exps = torch.zeros((3, groups), dtype=torch.uint8, device=d)
    s = qe.make_saved(qe.SAVED_I8, data, cols, exps, groups)
    assert qe.qe_act_save(x, q, cols, 3, cols, s) == "OK"
    codes, bytes_ = oa.pack(v)
    assert np.array_equal(data.cpu().numpy(), codes) and np.array_equal(exps.cpu().numpy(), bytes_)
    assert bytes_[0, 0] == 249 and np.abs(codes[0]).max() == 63
    back = torch.zeros_like(x)
    assert qe.qe_act_restore(s, 3, cols, back, q, cols) == "OK"
    off = np.abs(back.double().cpu().numpy() - v)
    assert (off < TOP).all() and (off[np.abs(v) < 63.5 * TOP] <= TOP / 2).all()


@pytest.mark.parametrize("shape", [(3, 40), (20, 130), (70, 300)], ids=str)
@pytest.mark.parametrize("tile", ["TILE_AUTO", "TILE_256x256"])
def test_products_save_the_largest_finite_values(tile, shape):
    """Pre-activations of a product (sums of nothing plus a bias) through each of its epilogues' checkpoints."""
    qe, d = need_lib(), dev()
    m, n = shape
    bias = np.zeros(n, dtype=np.float32)
    bias[:len(TOPMOST)] = TOPMOST
    bias[n - 1] = -LARGEST
    codes, one = torch.full((max(m, n), 16), 0x38, dtype=torch.uint8, device=d), torch.ones(1, device=d)
    groups = -(-n // 32)
    data = torch.zeros((m, n), dtype=torch.int8, device=d)
    exps = torch.zeros((m, groups), dtype=torch.uint8, device=d)
    c, b = torch.zeros((m, n), device=d), torch.from_numpy(bias).to(d)
    epi = qe.make_epilogue(bias=b, bias_dtype=qe.F32, saved=qe.make_saved(qe.SAVED_I8, data, n, exps, groups))
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        assert qe.qe_fp8_gemm_act(codes, 0, 16, codes, 0, 16, m, n, 0, one, one, epi, c, qe.F32, n) == "OK"
        torch.cuda.synchronize()
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"
    want = oa.pack(np.broadcast_to(bias, (m, n)))
    assert np.array_equal(data.cpu().numpy(), want[0]) and np.array_equal(exps.cpu().numpy(), want[1])
    assert np.isfinite(oa.unpack(*want).astype(np.float32)).all()
