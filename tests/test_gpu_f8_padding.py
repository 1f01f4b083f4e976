"""What a row of 8-bit codes has between its last element and a multiple of 128 is zero whatever the block holds, NaN among it: every call writes it so, and the products rely on it."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests.f8_device import FORMATS, Matrix, same
from tests.test_gpu_f8_quantize import source
from tests.test_gpu_train_mx import DTYPES

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (3, 127), (17, 513), (127, 129), (129, 255), (300, 1000), (130, 4)]


def spoiled(rows, cols, seed):
    """The last element of every row, and the last row, are no numbers: every block that padding belongs to is NaN, by rows and by columns."""
    x = np.random.default_rng(seed).standard_normal((rows, cols)).astype(np.float32)
    x[:, -1] = np.resize([np.nan, np.inf, -np.inf, -np.nan], rows)
    x[-1] = np.resize([np.inf, -np.nan, np.nan], cols)
    return x


def check(m, x, block_rows):
    codes, scales = m.read()
    assert not codes[:, m.cols:].any()
    assert np.all(np.isnan(scales[-1])) and same((codes, scales), fo.quantize(x, m.fmt, block_rows))


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_conversion(dtype, fmt, block_rows):
    for k, (rows, cols) in enumerate(SIZES):
        for which in ("rows", "columns", "both"):
            print(f"padding of {rows} x {cols} {dtype} {fmt} block_rows {block_rows} {which}", flush=True)
            x = spoiled(rows, cols, k)
            stored = x if dtype == "f32" else to.half_bits(x, dtype)
            seen = x if dtype == "f32" else to.half_values(stored, dtype).astype(np.float32)
            buf, at = source(stored, cols + k % 3, k % 2)
            by_row = Matrix(FORMATS[fmt], rows, cols, block_rows, wider=k % 2) if which != "columns" else None
            by_col = Matrix(FORMATS[fmt], cols, rows, block_rows, wider=k % 3) if which != "rows" else None
            B.f8_quantize(at, DTYPES[dtype][0], cols + k % 3, by_row and by_row.matrix, by_col and by_col.matrix, 0)
            harness.synchronize()
            if by_row:
                check(by_row, seen, block_rows)
            if by_col:
                check(by_col, seen.T, block_rows)
            del buf


@pytest.mark.parametrize("to_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_columns(fmt, to_fmt):
    for k, (rows, cols) in enumerate(SIZES):
        print(f"padding of columns {rows} x {cols} {fmt} to {to_fmt}", flush=True)
        held = fo.quantize(spoiled(rows, cols, k), FORMATS[fmt])
        src, dst = Matrix(FORMATS[fmt], rows, cols, held=held, wider=k % 3), Matrix(FORMATS[to_fmt], cols, rows, wider=k % 2)
        B.f8_columns(src.matrix, dst.matrix, 0)
        harness.synchronize()
        with np.errstate(all="ignore"):
            v = (fo.TABLE[FORMATS[fmt]][held[0]].astype(np.float32) * np.repeat(held[1].T, 128, 1))[:, :cols]
        check(dst, v.T, 1)
