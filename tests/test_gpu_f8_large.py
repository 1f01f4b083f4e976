"""Matrices whose codes, scales' places or results lie beyond 32-bit offsets: zero but for their last rows (and the last columns of what is read), looked at where those are."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu

ONE = int(fo.nearest_codes(np.ones(1), fo.E4M3)[0])


class Large:
    """rows x cols, all codes `byte`, all scales `scale`."""

    def __init__(self, rows, cols, byte=0, scale=1.0, fmt=fo.E4M3, block_rows=1, pitch=None):
        self.rows, self.cols, self.fmt = rows, cols, fmt
        self.pitch, self.scale_pitch = B.f8_layout(fmt, rows, cols, block_rows)
        self.pitch = pitch or self.pitch
        self.codes, self.scales = harness.DevBuf(rows * self.pitch), harness.DevBuf(4 * (fo.padded(cols) // 128) * self.scale_pitch)
        B.proxy_device_fill_async(self.codes.ptr, byte, self.codes.nbytes, 0)
        ones = np.full(self.scales.nbytes // 4, scale, np.float32)
        self.scales.upload(ones)
        self.matrix = B.f8_matrix(fmt, rows, cols, self.codes.ptr, self.pitch, self.scales.ptr, self.scale_pitch, block_rows)

    def put(self, row, codes):
        codes = np.ascontiguousarray(codes, np.uint8)
        harness.synchronize()
        B.proxy_copy_h2d(self.codes.ptr + row * self.pitch, codes.ctypes.data, codes.size)

    def row(self, row, first=0, count=None):
        return gu.download(self.codes, row * self.pitch + first, count or self.pitch)

    def scale(self, row, col):
        return float(gu.download(self.scales, 4 * ((col // 128) * self.scale_pitch + row), 4).view(np.float32)[0])


def test_conversion():
    n = 70000
    print("conversion of 70,000 x 70,000 bf16", flush=True)
    src = harness.DevBuf(2 * n * n)
    B.proxy_device_fill_async(src.ptr, 0, src.nbytes, 0)
    harness.synchronize()
    last = to.half_bits(np.linspace(-3, 5, n).astype(np.float32), "bf16")
    B.proxy_copy_h2d(src.ptr + 2 * (n - 1) * n, last.ctypes.data, last.nbytes)
    by_row, by_col = Large(n, n, 0xEE), Large(n, n, 0xEE)
    B.f8_quantize(src.ptr, B.CKPT_BF16, n, by_row.matrix, by_col.matrix, 0)
    again = Large(n, n, 0xEE)
    B.f8_columns(by_col.matrix, again.matrix, 0)
    B.f8_dequantize(by_row.matrix, src.ptr, B.CKPT_BF16, n, 0)
    harness.synchronize()
    x = to.half_values(last, "bf16").astype(np.float32)
    codes, scales = fo.quantize(x[None], fo.E4M3)
    assert np.array_equal(by_row.row(n - 1), codes[0]) and not by_row.row(n - 2).any() and by_row.scale(n - 1, n - 1) == scales[-1, 0]
    col_codes, col_scales = fo.quantize(np.concatenate([np.zeros((1, n - 1), np.float32), x[None, -1:]], 1), fo.E4M3)      # the last column's block holds one value
    assert np.array_equal(by_col.row(n - 1), col_codes[0]) and by_col.scale(n - 1, n - 1) == col_scales[-1, 0]
    with np.errstate(all="ignore"):
        twice = (448 * np.maximum(np.abs(x) / np.float32(448), np.float32(2.0 ** -126))).astype(np.float32) * np.sign(x)      # a block's only value is its largest
    assert np.allclose(fo.values(again.row(n - 1)[None], np.array([[again.scale(n - 1, c)] for c in range(0, n, 128)]), fo.E4M3, n)[0], twice, rtol=2.0 ** -4 + 1e-6, atol=np.abs(x).max() / 448 * 2.0 ** -10)
    back = to.half_values(gu.download(src, 2 * (n - 1) * n, 2 * n).view(np.uint16), "bf16")
    want = fo.values(codes, scales, fo.E4M3, n)[0]
    assert np.all(np.abs(back - want) <= 2.0 ** -8 * np.abs(want))


@pytest.mark.parametrize("m", [3, 50])
def test_product(m):
    n, k = 40000, 131072
    print(f"product {m} x {n} x {k}", flush=True)
    a, b = Large(m, k, ONE), Large(n, k)
    b.put(n - 2, np.full(k, ONE))
    c = harness.DevBuf(4 * n * m)
    B.f8_gemm(a.matrix, b.matrix, c.ptr, B.CKPT_F32, n, 0)
    harness.synchronize()
    got = gu.download(c).view(np.float32).reshape(m, n)
    want = np.zeros((m, n), np.float32)
    want[:, n - 2] = k
    assert np.array_equal(got, want)
    B.f8_gemm(b.matrix, a.matrix, c.ptr, B.CKPT_F32, m, 0)          # more than 4 GiB on the other side
    harness.synchronize()
    assert np.array_equal(gu.download(c).view(np.float32).reshape(n, m), want.T)


def test_gated_block():
    t, d, f = 400000, 128, 11008
    print(f"gated block of {t} tokens, {d} to {f}", flush=True)
    x, w = Large(t, d), [Large(f, d, ONE, 1 / 128, block_rows=128) for _ in range(3)]
    x.put(t - 1, np.full(d, ONE))
    gate, up, h = (Large(t, f, 0xEE) for _ in range(3))
    B.gated_forward(x.matrix, w[0].matrix, w[1].matrix, B.CKPT_GATE_SILU, 0, h.matrix, gate.matrix, up.matrix)
    grads = {k: Large(t, f, 0xEE) for k in ("dgate", "dup")} | {k: Large(f, t, 0xEE) for k in ("dgate_by_col", "dup_by_col", "h_by_col")}
    B.gated_backward(x.matrix, w[2].matrix, gate.matrix, up.matrix, B.CKPT_GATE_SILU, 0, **{k: v.matrix for k, v in grads.items()})
    harness.synchronize()
    # gate = up = dh = 1 at the last token, zero elsewhere
    s = 1 / (1 + np.exp(-1.0))
    for m, value in ((gate, 1.0), (up, 1.0), (h, s), (grads["dgate"], s * (2 - s)), (grads["dup"], s)):
        assert np.all(m.row(t - 1) == 0x7E) and not m.row(t - 2).any() and abs(m.scale(t - 1, f - 1) * 448 - value) < 1e-6
    for k, value in (("dgate_by_col", s * (2 - s)), ("dup_by_col", s), ("h_by_col", s)):
        last = grads[k].row(f - 1)
        assert last[t - 1] == 0x7E and not last[: t - 1].any() and abs(grads[k].scale(f - 1, t - 1) * 448 - value) < 1e-6


def test_columns_in_the_longest_rows():
    t, d, f = 40, 128, 200
    print("backward pass, columns' forms in rows of 2^23 bytes", flush=True)
    rng = np.random.default_rng(5)
    dy, w, gate, up = Large(t, d), Large(f, d), Large(t, f), Large(t, f)
    for m in (dy, w, gate, up):
        for r in range(m.rows):
            m.put(r, np.concatenate([fo.nearest_codes(rng.standard_normal(m.cols), fo.E4M3), np.zeros(-m.cols % 128)]))
    given = dy.matrix, w.matrix, gate.matrix, up.matrix, B.CKPT_GATE_SILU, 0
    forms = "dgate_by_col", "dup_by_col", "h_by_col"
    plain = {k: Large(f, t, 0xEE) for k in forms}
    B.gated_backward(*given, **{k: v.matrix for k, v in plain.items()})
    for k in forms:
        far = Large(f, t, 0xEE, pitch=1 << 23)
        B.gated_backward(*given, **{k: far.matrix})
        harness.synchronize()
        for r in range(f):
            assert np.array_equal(far.row(r, 0, 128), plain[k].row(r)) and np.all(far.row(r, 128, 128) == 0xEE), (k, r)
            assert far.scale(r, 0) == plain[k].scale(r, 0)
            assert plain[k].row(r)[:t].any()
