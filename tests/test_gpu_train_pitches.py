"""The block-scaled operators where rows lie further apart than they have to, and products on the routes that only such rows, a small workspace or none lead to. Products are exact: see
test_gpu_train_gemm.py."""
import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu
from tests.test_gpu_train_gemm import exactly, on_device, operand
from tests.test_gpu_train_mx import DTYPES, content, guarded, inputs

pytestmark = pytest.mark.gpu

LONGEST = 1 << 23      # bytes from row to row that the tile kernels take


class Operand:
    """codes [rows, k] and their scales in rows of given pitches, zeros behind them."""

    def __init__(self, codes, byte, code_pitch, scale_pitch):
        rows, k = codes.shape
        self.bufs = []
        for part, pitch in zip(to.pack_rows(codes, byte, to.MXFP4, -(-k // 256) * 128, -(-k // 32)), (code_pitch, scale_pitch)):
            buf = harness.DevBuf(rows * pitch)
            B.proxy_device_fill_async(buf.ptr, 0, buf.nbytes, 0)
            harness.synchronize()
            for r in range(rows):
                row = np.ascontiguousarray(part[r])
                B.proxy_copy_h2d(buf.ptr + r * pitch, row.ctypes.data, row.nbytes)
            self.bufs.append(buf)
        self.mx = B.mx_matrix(to.MXFP4, rows, k, self.bufs[0].ptr, code_pitch, self.bufs[1].ptr, scale_pitch)

    def free(self):
        for b in self.bufs:
            b.free()


def check_product(ma, mb, want, out, accumulate, pad, workspace_bytes=0):
    """want: float64 [m, n], exact; twice, for the same bits."""
    m, n = want.shape
    size, ldc = (4 if out == "f32" else 2), n + pad
    before = np.random.default_rng(7).integers(-64, 65, (m, ldc)).astype(np.float32)
    stored = before if out == "f32" else to.half_bits(before, "bf16")
    nbytes = (m * ldc - pad) * size
    ws = harness.DevBuf(max(workspace_bytes, 16) + 256)
    want = exactly(want + before[:, :n] if accumulate else want, out)
    for _ in range(2):
        held, ptr = guarded(nbytes, stored.tobytes()[:nbytes], 0)
        ws.upload(np.full(ws.nbytes, 0xFF, np.uint8))
        B.mx_gemm(ma, mb, ptr, B.CKPT_F32 if out == "f32" else B.CKPT_BF16, ldc, 0, accumulate=accumulate, workspace=ws.ptr if workspace_bytes else None, workspace_bytes=workspace_bytes)
        harness.synchronize()
        raw = np.concatenate([content(held, nbytes), np.frombuffer(stored.tobytes()[nbytes:], np.uint8)]).view(stored.dtype).reshape(m, ldc)
        assert np.array_equal(raw[:, n:], stored[:, n:])
        assert np.array_equal(raw[:, :n].astype(np.float64) if out == "f32" else to.half_values(raw[:, :n], "bf16"), want)
        assert np.all(gu.download(ws)[workspace_bytes:] == 0xFF), "written behind the workspace"


def exact(a, b):
    want, magnitude = to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))
    assert magnitude.max() + 64 < 2.0 ** 22
    return want


@pytest.mark.parametrize("out,accumulate", [("bf16", False), ("f32", False), ("f32", True), ("bf16", True)])
@pytest.mark.parametrize("m,n,k", [(17, 33, 300), (130, 70, 1000), (64, 128, 256), (40, 20, 4097)])
def test_rows_too_long_for_the_tiles(m, n, k, out, accumulate):
    print(f"product {m} x {n} x {k}, rows of more than 2^23 bytes, {out}, accumulate {accumulate}", flush=True)
    rng = np.random.default_rng(m)
    a, b = operand(m, k, rng, 1), operand(n, k, rng, 1)
    want = exact(a, b)
    cp, sp = B.mx_layout(to.MXFP4, 1, k)
    longer = LONGEST + 128
    for pitches_a, pitches_b in (((longer, -(-longer // 256) * 16), (longer, -(-longer // 256) * 16)), ((cp, sp), (longer, -(-longer // 256) * 16)), ((cp, LONGEST + 16), (cp, sp))):
        x, y = Operand(*a, *pitches_a), Operand(*b, *pitches_b)
        check_product(x.mx, y.mx, want, out, accumulate, 3 * (m % 2))
        x.free()
        y.free()


def test_an_axis_too_long_for_the_tiles():
    """K of 2^24 + 300 and more: zeros but for some blocks, the first and the last among them."""
    m, n, k = 18, 35, (1 << 24) + 300
    print(f"product {m} x {n} x {k}", flush=True)
    rng = np.random.default_rng(4)
    blocks = np.concatenate([[0, 1, 31], rng.integers(32, k // 32, 60), [k // 32 - 1, k // 32]])
    cp, sp = B.mx_layout(to.MXFP4, m, k)
    assert cp > LONGEST
    values, mats, held = [], [], []
    for rows in (m, n):
        codes, byte = operand(rows, 32 * len(blocks), rng, 1)
        codes[:, 32 * len(blocks) - 32 + k % 32:] = 0
        values.append(to.values(codes, byte, to.MXFP4))
        c, s = harness.DevBuf(rows * cp), harness.DevBuf(rows * sp)
        for buf in (c, s):
            B.proxy_device_fill_async(buf.ptr, 0, buf.nbytes, 0)
        harness.synchronize()
        host_c, host_s = np.zeros(cp, np.uint8), np.zeros(sp, np.uint8)
        for r in range(rows):
            for j, block in enumerate(blocks):
                part = codes[r, 32 * j:32 * j + 32]
                host_c[16 * block:16 * block + 16] = part[0::2] | (part[1::2] << 4)
                host_s[block] = byte[r, j]
            B.proxy_copy_h2d(c.ptr + r * cp, host_c.ctypes.data, cp)
            B.proxy_copy_h2d(s.ptr + r * sp, host_s.ctypes.data, sp)
        held += [c, s]
        mats.append(B.mx_matrix(to.MXFP4, rows, k, c.ptr, cp, s.ptr, sp))
    # a block that was drawn twice holds what was put there last
    last = {int(b): j for j, b in enumerate(blocks)}
    keep = np.repeat([last[int(b)] == j for j, b in enumerate(blocks)], 32)
    want, magnitude = to.gemm(values[0] * keep, values[1] * keep)
    assert magnitude.max() + 64 < 2.0 ** 22
    check_product(mats[0], mats[1], want, "f32", False, 1)
    for x in held:
        x.free()


@pytest.mark.parametrize("wider,wider_scales", [(128, 0), (0, 16), (256, 48)])
@pytest.mark.parametrize("m,n,k", [(1, 100, 300), (16, 70, 5000), (1000, 2304, 768), (500, 1030, 2000), (300, 200, 512), (130, 100, 20000), (2000, 2050, 1030)])
def test_rows_further_apart_than_they_have_to_be(m, n, k, wider, wider_scales):
    print(f"product {m} x {n} x {k}, pitches {wider} and {wider_scales} wider", flush=True)
    rng = np.random.default_rng(n)
    a, b = operand(m, k, rng, 0), operand(n, k, rng, 0)
    want = exact(a, b)
    cp, sp = B.mx_layout(to.MXFP4, 1, k)
    scale_pitch = -(-(cp + wider) // 256) * 16
    x, y = Operand(*a, cp + wider, scale_pitch + wider_scales), Operand(*b, cp, sp)
    for out in ("f32", "bf16"):
        check_product(x.mx, y.mx, want, out, False, 0, B.mx_gemm_workspace(m, n, k))
        check_product(y.mx, x.mx, want.T, out, True, 2, B.mx_gemm_workspace(n, m, k))


@pytest.mark.parametrize("out,accumulate", [("bf16", True), ("f32", False)])
@pytest.mark.parametrize("m,n,k", [(17, 64, 16384), (64, 512, 16384), (130, 100, 20000), (30, 1001, 16000)])
def test_a_workspace_for_some_of_the_parts(m, n, k, out, accumulate):
    whole = B.mx_gemm_workspace(m, n, k)
    part = m * -(-n // 4) * 16
    assert whole >= 4 * part
    rng = np.random.default_rng(k)
    a, b = operand(m, k, rng, 0), operand(n, k, rng, 0)
    want = exact(a, b)
    _, ma = ha = on_device(*a)
    _, mb = hb = on_device(*b)
    for nbytes in (whole - 16, whole // 2, 2 * part, 2 * part - 16, part, 16, 0):
        print(f"product {m} x {n} x {k} in parts, {nbytes} of {whole} bytes", flush=True)
        check_product(ma, mb, want, out, accumulate, 1, nbytes // 16 * 16)


@pytest.mark.parametrize("m,n,k", [(1, 64, 300), (16, 100, 4100), (100, 130, 520), (300, 520, 1024)])
def test_scales_from_one_end_to_the_other(m, n, k):
    """Scales from 2^-127 to 2^127 a row: exact where f32 holds the result as a normal number, infinite above, at most its smallest normal number below."""
    print(f"product {m} x {n} x {k}, all scales", flush=True)
    rng = np.random.default_rng(9)
    exponents = np.array([-127, -126, -100, -64, -10, 0, 10, 64, 100, 126, 127])
    rows = [rng.choice(exponents, r) for r in (m, n)]
    codes = [rng.integers(1, 8, (r, k)).astype(np.uint8) for r in (m, n)]      # 0.5 to 6
    a, b = ((c, np.repeat((127 + e)[:, None], -(-k // 32), axis=1).astype(np.uint8)) for c, e in zip(codes, rows))
    plain, magnitude = to.gemm(to.FP4[codes[0]], to.FP4[codes[1]])
    assert magnitude.max() < 2.0 ** 22
    want = plain * 2.0 ** (rows[0][:, None] + rows[1][None, :]).astype(np.float64)
    held_a, ma = on_device(*a)
    held_b, mb = on_device(*b)
    held, ptr = guarded(m * n * 4)
    B.mx_gemm(ma, mb, ptr, B.CKPT_F32, n, 0)
    harness.synchronize()
    got = content(held, m * n * 4).view(np.float32).reshape(m, n)
    above, below = want >= 2.0 ** 128, want < 2.0 ** -126
    assert above.any() == (want.max() >= 2.0 ** 128) and np.all(np.isposinf(got[above]))
    assert np.all((got[below] >= 0) & (got[below] <= 2.0 ** -126))
    assert np.array_equal(got[~above & ~below].astype(np.float64), want[~above & ~below])


def quantized(stored, dtype, rows, cols, fmt, pitches, rounding, seed):
    """by_row and, if pitches has a second pair, by_col; what was in the memory before is 0xEE."""
    held, ptr = guarded(stored.nbytes, stored.tobytes())
    outs, mats = [], []
    for (r, c), (cp, sp) in zip(((rows, cols), (cols, rows)), pitches):
        codes, cptr = guarded(r * cp)
        scales, sptr = guarded(r * sp)
        outs.append((codes, r, cp, scales, sp))
        mats.append(B.mx_matrix(fmt, r, c, cptr, cp, sptr, sp))
    B.mx_quantize(ptr, DTYPES[dtype][0], cols, mats[0], mats[1] if len(mats) > 1 else None, 0, rounding=rounding, seed=seed)
    harness.synchronize()
    return mats, [(content(c, r * cp).reshape(r, cp), content(s, r * sp).reshape(r, sp)) for c, r, cp, s, sp in outs], outs


@pytest.mark.parametrize("rounding", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_mxfp8_from_every_type_in_wider_rows(dtype, rounding):
    for k, (rows, cols, wider, wider_scales) in enumerate([(1, 1, 0, 0), (1, 33, 5, 0), (3, 97, 1, 2), (40, 100, 31, 0), (5, 1000, 24, 3), (2, 5001, 1100, 40), (300, 7, 0, 1), (1, 70000, 0, 0)]):
        print(f"fp8 {dtype} rounding {rounding} {rows} x {cols}, {wider} and {wider_scales} wider", flush=True)
        stored, x = inputs(rows, cols, dtype, 900 + k, special=k % 2 == 1)
        pitch, scale_pitch = cols + wider, -(-cols // 32) + wider_scales
        _, got, _ = quantized(stored, dtype, rows, cols, to.MXFP8, [(pitch, scale_pitch)], rounding, 40 + k)
        codes, byte = to.quantize(x, to.MXFP8, int(to.mix(np.uint64(40 + k))) if rounding & 1 else None, bool(rounding & 2))
        want, scales = to.pack_rows(codes, byte, to.MXFP8, pitch, scale_pitch)
        assert np.array_equal(got[0][1], scales)
        nan = np.zeros(want.shape, bool)
        nan[:, :cols] = np.repeat(byte == 255, 32, axis=1)[:, :cols]
        assert np.array_equal(got[0][0][~nan], want[~nan])


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_mxfp4_in_wider_rows_and_back(dtype, rounding):
    for k, (rows, cols, wider, wider_scales) in enumerate([(1, 1, 128, 0), (3, 128, 128, 16), (130, 513, 256, 0), (5, 1030, 0, 32), (64, 256, 1024, 64)]):
        for both in (False, True):
            print(f"fp4 {dtype} rounding {rounding} {rows} x {cols}, {wider} and {wider_scales} wider, both forms {both}", flush=True)
            stored, x = inputs(rows, cols, dtype, 950 + k, special=k % 2 == 1)
            pitches = []
            for r, c in ((rows, cols), (cols, rows))[: 1 + both]:
                pitch = B.mx_layout(to.MXFP4, r, c)[0] + wider
                pitches.append((pitch, -(-pitch // 256) * 16 + wider_scales))
            mats, got, _outs = quantized(stored, dtype, rows, cols, to.MXFP4, pitches, rounding, 60 + k)
            keys = [int(to.mix(np.uint64(s & to.U64))) if rounding else None for s in (60 + k, ~(60 + k))]
            for y, key, mat, (got_codes, got_scales), (pitch, scale_pitch) in zip((x, x.T), keys, mats, got, pitches):
                codes, byte = to.quantize(y, to.MXFP4, key)
                want, scales = to.pack_rows(codes, byte, to.MXFP4, pitch, scale_pitch)
                assert np.array_equal(got_scales, scales)
                nan = np.zeros(want.shape, bool)
                at = np.repeat(byte == 255, 16, axis=1)[:, :pitch]
                nan[:, : at.shape[1]] = at
                assert np.array_equal(got_codes[~nan], want[~nan])
                r, c = y.shape
                held, ptr = guarded(r * c * 4)
                B.mx_dequantize(mat, ptr, B.CKPT_F32, c, 0)
                harness.synchronize()
                back = content(held, r * c * 4).view(np.float32).reshape(r, c)
                value = to.values(codes, byte, to.MXFP4)
                assert np.array_equal(np.isnan(back), np.isnan(value)) and np.array_equal(back[~np.isnan(value)], value[~np.isnan(value)])
