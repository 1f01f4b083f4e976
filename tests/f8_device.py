"""Matrices in 8 bits on the device, between guards, for the GPU tests of the operators with blocks of 128."""
import numpy as np

from oracle import f8_oracle as fo
from paper_2406_10707_amd import binding as B
from tests.test_gpu_train_mx import content, guarded

FORMATS = {"e4m3": fo.E4M3, "e5m2": fo.E5M2}


class Matrix:
    """rows x cols with memory of its own; `wider`: that many pieces of 16 bytes, and scales, more from row to row."""

    def __init__(self, fmt, rows, cols, block_rows=1, held=None, wider=0):
        self.fmt, self.rows, self.cols, self.block_rows = fmt, rows, cols, block_rows
        self.code_pitch, self.scale_pitch = fo.padded(cols) + 16 * wider, -(-rows // block_rows) + wider
        self.code_bytes = max(0, (rows - 1) * self.code_pitch + fo.padded(cols)) if rows and cols else 0
        blocks = fo.padded(cols) // 128
        self.scale_count = max(0, (blocks - 1) * self.scale_pitch + -(-rows // block_rows)) if rows and cols else 0
        codes, scales = np.full(rows * self.code_pitch, 0xEE, np.uint8), np.full(blocks * self.scale_pitch, -7.0, np.float32)
        if held is not None:
            codes.reshape(rows, -1)[:, : fo.padded(cols)] = held[0]
            scales.reshape(blocks, -1)[:, : -(-rows // block_rows)] = held[1]
        # the guards begin right behind the last byte that belongs to the matrix; 16-byte aligned, as the guards' own size is
        self.codes = guarded(self.code_bytes, codes.tobytes()[: self.code_bytes])
        self.scales = guarded(4 * self.scale_count, scales.tobytes()[: 4 * self.scale_count])
        self.matrix = B.f8_matrix(fmt, rows, cols, self.codes[1], self.code_pitch, self.scales[1], self.scale_pitch, block_rows)

    def read(self):
        """(codes, scales), as the oracle has them; what lies between rows is as it was."""
        codes = np.concatenate([content(self.codes[0], self.code_bytes), np.full(self.rows * self.code_pitch - self.code_bytes, 0xEE, np.uint8)]).reshape(self.rows, -1)
        blocks, count = fo.padded(self.cols) // 128, -(-self.rows // self.block_rows)
        raw = content(self.scales[0], 4 * self.scale_count).view(np.float32)
        scales = np.concatenate([raw, np.full(blocks * self.scale_pitch - self.scale_count, -7.0, np.float32)]).reshape(blocks, -1)
        assert np.all(codes[:, fo.padded(self.cols):] == 0xEE), "written between rows"
        between = scales[:, count:]
        assert np.all((between == -7.0) | (between.view(np.uint32) == 0xEEEEEEEE)), "written between blocks of scales"
        return codes[:, : fo.padded(self.cols)], scales[:, :count]

    def values(self):
        return fo.values(*self.read(), self.fmt, self.cols, self.block_rows)


def same(got, want):
    """Bit for bit, codes of blocks whose scale is NaN apart."""
    codes, scales = got
    if not np.array_equal(scales, want[1], equal_nan=True):
        return False
    rows = codes.shape[0]
    nan = np.repeat(np.repeat(np.isnan(scales).T, 128 if scales.shape[1] < rows else 1, 0)[:rows], 128, 1)
    return np.array_equal(codes[~nan], want[0][~nan])
