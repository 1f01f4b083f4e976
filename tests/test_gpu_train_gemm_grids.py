"""Products whose C takes more than one grid: each launch writes its own part, and the parts meet."""
import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu
from tests.test_gpu_train_gemm import exactly, on_device, operand

pytestmark = pytest.mark.gpu


def test_more_columns_than_a_grid_of_few_rows():
    """Up to 2^27 columns are a launch's. B is ones but for its first rows, those around the border and its last."""
    m, n, k = 3, (1 << 27) + 1000, 200
    print(f"product {m} x {n} x {k}", flush=True)
    rng = np.random.default_rng(1)
    a = operand(m, k, rng, 1)
    _held, ma = on_device(*a)
    cp, sp = B.mx_layout(to.MXFP4, n, k)
    codes, scales, c = harness.DevBuf(n * cp), harness.DevBuf(n * sp), harness.DevBuf(m * n * 2)
    ones = to.pack_rows(np.full((1 << 16, k), 2, np.uint8), np.full((1 << 16, 7), 127, np.uint8), to.MXFP4, cp, sp)
    for part, buf in zip(ones, (codes, scales)):
        B.proxy_copy_h2d(buf.ptr, part.ctypes.data, part.nbytes)
        for at in range(part.nbytes, buf.nbytes, part.nbytes):
            B.proxy_copy_d2d_async(buf.ptr + at, buf.ptr, min(part.nbytes, buf.nbytes - at), 0)
    harness.synchronize()
    b = operand(64, k, rng, 1)
    pc, ps = to.pack_rows(*b, to.MXFP4, cp, sp)
    places = (0, (1 << 27) - 32, n - 64)
    for at in places:
        B.proxy_copy_h2d(codes.ptr + at * cp, pc.ctypes.data, pc.nbytes)
        B.proxy_copy_h2d(scales.ptr + at * sp, ps.ctypes.data, ps.nbytes)
    B.proxy_device_fill_async(c.ptr, 0xEE, c.nbytes, 0)
    B.mx_gemm(ma, B.mx_matrix(to.MXFP4, n, k, codes.ptr, cp, scales.ptr, sp), c.ptr, B.CKPT_BF16, n, 0)
    harness.synchronize()
    values = to.values(*a, to.MXFP4)
    want, plain = exactly(to.gemm(values, to.values(*b, to.MXFP4))[0], "bf16"), exactly(values.sum(1, keepdims=True), "bf16")
    for row in range(m):
        got = gu.download(c, 2 * row * n, 2 * n).view(np.uint16)
        for at in places:
            assert np.array_equal(to.half_values(got[at:at + 64], "bf16"), want[row])
            got[at:at + 64] = to.half_bits(plain[row].astype(np.float32), "bf16")
        assert np.all(got == got[0])
    for x in (codes, scales, c):
        x.free()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_no_columns_and_more_rows_than_a_grid(out, accumulate):
    m, n = 65535 * 64 + 500, 3
    print(f"product {m} x {n} x 0, {out}, accumulate {accumulate}", flush=True)
    size = 4 if out == "f32" else 2
    c = harness.DevBuf(m * n * size + 64)
    before = np.full(c.nbytes, 0x11, np.uint8)
    c.upload(before)
    a, b = (B.mx_matrix(B.CKPT_MXFP4, r, 0, None, 0, None, 0) for r in (m, n))
    B.mx_gemm(a, b, c.ptr, B.CKPT_F32 if out == "f32" else B.CKPT_BF16, n, 0, accumulate=accumulate)
    harness.synchronize()
    got = gu.download(c)
    assert np.all(got[-64:] == 0x11) and np.all(got[:-64] == (0x11 if accumulate else 0))
