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
