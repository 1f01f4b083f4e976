"""Conversion to 8 bits in blocks of 128, the columns' form of what is held in 8 bits, and back, against the oracle bit for bit: sizes from one element on, ragged rows, strides, unaligned starts, zeros, infinities, NaN,
ties, subnormal numbers; nothing outside the outputs is written."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests.f8_device import FORMATS, Matrix, same
from tests.test_gpu_train_mx import DTYPES, content, guarded

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 128), (3, 127), (16, 512), (17, 513), (1, 4096), (128, 128), (127, 129), (129, 255), (130, 384), (300, 1000), (1000, 40), (5, 8), (257, 257), (512, 1024)]


def inputs(rows, cols, dtype, seed):
    """As stored, and in f32: many magnitudes, ties of both formats, zero blocks, signed zeros, infinities, NaN, subnormal numbers."""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 7, (rows, cols))).astype(np.float32)
    x[rng.random((rows, cols)) < 0.1] = 0
    ties = rng.random((rows, cols)) < 0.3
    x[ties] = rng.choice([448.0, -448.0, 17 / 16, 19 / 16, 9 / 8, 11 / 8, 2.0 ** -10, 3 * 2.0 ** -10, -0.0, 5 * 2.0 ** -17], ties.sum())
    for r in range(rows):
        for b in range(0, cols, 128):
            u = rng.random()
            if u < 0.08:
                x[r, b:b + 128] = 0
            elif u < 0.12 and rows > 2:
                x[r, min(cols - 1, b + int(rng.integers(128)))] = rng.choice([np.inf, -np.inf, np.nan])
            elif u < 0.2:
                x[r, b:b + 128] *= np.float32(2.0 ** -130)
            elif u < 0.25 and dtype != "f16":
                x[r, b:b + 128] *= np.float32(2.0 ** 100)
    if dtype == "f32":
        return x, x
    with np.errstate(over="ignore"):
        bits = to.half_bits(x, dtype)
    return bits, to.half_values(bits, dtype).astype(np.float32)


def source(stored, ld, shift):
    """(buffer, address) of a row-major matrix with `ld` elements from row to row, `shift` elements behind an aligned address."""
    rows, cols = stored.shape
    wide = np.full((rows, ld), 0x7E, stored.dtype if stored.dtype != np.float32 else np.uint32)
    wide[:, :cols] = stored.view(wide.dtype)
    nbytes = ((rows - 1) * ld + cols) * wide.itemsize
    return guarded(nbytes, wide.tobytes()[:nbytes], shift * wide.itemsize)


@pytest.mark.parametrize("which", ["rows", "columns", "both"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quantize(dtype, fmt, block_rows, which):
    for k, (rows, cols) in enumerate(SIZES):
        print(f"quantize {rows} x {cols} {dtype} {fmt} block_rows {block_rows} {which}", flush=True)
        stored, x = inputs(rows, cols, dtype, 10 + k)
        buf, at = source(stored, cols + 3 * (k % 3), k % 3)
        by_row = Matrix(FORMATS[fmt], rows, cols, block_rows, wider=k % 2) if which != "columns" else None
        by_col = Matrix(FORMATS[fmt], cols, rows, block_rows, wider=k % 3) if which != "rows" else None
        B.f8_quantize(at, DTYPES[dtype][0], cols + 3 * (k % 3), by_row and by_row.matrix, by_col and by_col.matrix, 0)
        harness.synchronize()
        if by_row:
            assert same(by_row.read(), fo.quantize(x, FORMATS[fmt], block_rows))
        if by_col:
            assert same(by_col.read(), fo.quantize(x.T, FORMATS[fmt], block_rows))
        del buf


def test_two_formats_at_once():
    stored, x = inputs(200, 300, "f32", 3)
    buf, at = source(stored, 300, 0)
    by_row, by_col = Matrix(fo.E4M3, 200, 300), Matrix(fo.E5M2, 300, 200)
    B.f8_quantize(at, B.CKPT_F32, 300, by_row.matrix, by_col.matrix, 0)
    harness.synchronize()
    assert same(by_row.read(), fo.quantize(x, fo.E4M3)) and same(by_col.read(), fo.quantize(x.T, fo.E5M2))


@pytest.mark.parametrize("to_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_columns(fmt, to_fmt):
    for k, (rows, cols) in enumerate(SIZES):
        print(f"columns {rows} x {cols} {fmt} to {to_fmt}", flush=True)
        _, x = inputs(rows, cols, "f32", 40 + k)
        x = np.where(np.abs(x) > 1e30, x * np.float32(2.0 ** -60), x)      # else two bits of the larger format's products with the scale overflow
        held = fo.quantize(x, FORMATS[fmt])
        src, dst = Matrix(FORMATS[fmt], rows, cols, held=held, wider=k % 3), Matrix(FORMATS[to_fmt], cols, rows, wider=k % 2)
        B.f8_columns(src.matrix, dst.matrix, 0)
        harness.synchronize()
        with np.errstate(all="ignore"):
            v = (fo.TABLE[FORMATS[fmt]][held[0]].astype(np.float32) * np.repeat(held[1].T, 128, 1))[:, :cols]
        assert same(dst.read(), fo.quantize(v.T, FORMATS[to_fmt]))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_columns_of_square_blocks_are_the_same_values(fmt):
    rng = np.random.default_rng(5)
    for rows, cols in SIZES:
        print(f"columns of square blocks {rows} x {cols} {fmt}", flush=True)
        codes = np.zeros((rows, fo.padded(cols)), np.uint8)
        codes[:, :cols] = rng.integers(0, 256, (rows, cols))              # any code, NaN among them, moves as it is
        scales = rng.standard_normal((fo.padded(cols) // 128, -(-rows // 128))).astype(np.float32)
        src, dst = Matrix(FORMATS[fmt], rows, cols, 128, held=(codes, scales)), Matrix(FORMATS[fmt], cols, rows, 128)
        B.f8_columns(src.matrix, dst.matrix, 0)
        harness.synchronize()
        got = dst.read()
        want = np.zeros((cols, fo.padded(rows)), np.uint8)
        want[:, :rows] = codes[:, :cols].T
        assert np.array_equal(got[0], want) and np.array_equal(got[1], scales.T)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_dequantize(fmt, dtype, block_rows):
    for k, (rows, cols) in enumerate(SIZES):
        print(f"dequantize {rows} x {cols} {fmt} to {dtype} block_rows {block_rows}", flush=True)
        _, x = inputs(rows, cols, "f16", 70 + k)
        held = fo.quantize(x, FORMATS[fmt], block_rows)
        src = Matrix(FORMATS[fmt], rows, cols, block_rows, held=held, wider=k % 2)
        ld, size = cols + k % 4, DTYPES[dtype][1]
        nbytes = ((rows - 1) * ld + cols) * size
        buf, at = guarded(nbytes, shift=(k % 3) * size)
        B.f8_dequantize(src.matrix, at, DTYPES[dtype][0], ld, 0)
        harness.synchronize()
        raw = np.concatenate([content(buf, nbytes, (k % 3) * size), np.full((rows * ld) * size - nbytes, 0xEE, np.uint8)]).reshape(rows, -1)
        assert np.all(raw[:, cols * size:] == 0xEE)
        got = np.ascontiguousarray(raw[:, : cols * size])
        with np.errstate(all="ignore"):
            scale = np.repeat(np.repeat(held[1].T, block_rows, 0)[:rows], 128, 1)
            v = (fo.TABLE[FORMATS[fmt]][held[0]].astype(np.float32) * scale)[:, :cols]
            want = v if dtype == "f32" else to.half_values(to.half_bits(v, dtype), dtype)
        seen = got.view(np.float32) if dtype == "f32" else to.half_values(got.view(np.uint16), dtype)
        assert np.array_equal(seen, want, equal_nan=True)


def test_a_half_of_a_wider_matrix():
    """Columns 128 to 383 of a matrix 512 wide, as one that is written and one that is read."""
    stored, x = inputs(70, 256, "bf16", 8)
    buf, at = source(stored, 256, 0)
    whole = Matrix(fo.E4M3, 70, 512)
    part = B.f8_matrix(fo.E4M3, 70, 256, whole.codes[1] + 128, 512, whole.scales[1] + 4 * whole.scale_pitch, whole.scale_pitch)
    B.f8_quantize(at, B.CKPT_BF16, 256, part, None, 0)
    out = Matrix(fo.E4M3, 256, 70)
    B.f8_columns(part, out.matrix, 0)
    harness.synchronize()
    codes, scales = content(whole.codes[0], whole.code_bytes).reshape(70, 512), content(whole.scales[0], 4 * whole.scale_count).view(np.float32).reshape(4, 70)
    want = fo.quantize(x, fo.E4M3)
    assert np.all(codes[:, :128] == 0xEE) and np.all(codes[:, 384:] == 0xEE) and same((codes[:, 128:384], scales[1:3]), want)
    with np.errstate(all="ignore"):
        v = fo.TABLE[fo.E4M3][want[0]].astype(np.float32) * np.repeat(want[1].T, 128, 1)
    assert same(out.read(), fo.quantize(v.T, fo.E4M3))
