"""The product of two matrices in 8 bits with a scale for each block of 128. Codes stand for small whole numbers and scales are powers of two, so that every partial sum is a multiple of the smallest product that 24 bits
hold: f32 sums are then exact in any order, and the result is compared bit for bit. One test with real data has the bound that f32 accumulation gives."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu
from tests.f8_device import FORMATS, Matrix
from tests.test_gpu_train_mx import DTYPES, content, guarded

pytestmark = pytest.mark.gpu


def operand(fmt, rows, cols, block_rows, rng, spread=1):
    """(codes, scales): whole numbers up to 3, scales 2^0 .. 2^spread."""
    codes = np.zeros((rows, fo.padded(cols)), np.uint8)
    codes[:, :cols] = fo.nearest_codes(rng.integers(-3, 4, (rows, cols)).astype(np.float64), fmt)
    return codes, (2.0 ** rng.integers(0, spread + 1, (fo.padded(cols) // 128, -(-rows // block_rows)))).astype(np.float32)


def product(a, b, out, accumulate=False, pad=0, shift=0, workspace=True, rng=None, seed_c=0):
    """(result, C before) as float64, after two calls that give the same bits."""
    m, n, k = a.rows, b.rows, a.cols
    code, size = DTYPES[out]
    ldc = n + pad
    before = np.random.default_rng(seed_c).integers(-64, 65, (m, ldc)).astype(np.float32)
    stored = before if out == "f32" else to.half_bits(before, out)
    nbytes = (m * ldc - pad) * size
    hc, at = guarded(nbytes, stored.tobytes()[:nbytes], shift * size)
    need = B.f8_gemm_workspace(m, n, k) if workspace else 0
    ws = harness.DevBuf(max(need, 16))
    ws.upload(np.full(ws.nbytes, 0xFF, np.uint8))       # its contents do not matter
    first = None
    for _ in range(2):
        B.proxy_copy_h2d(at, stored.ctypes.data, nbytes)
        B.f8_gemm(a.matrix, b.matrix, at, code, ldc, 0, accumulate=accumulate, workspace=ws.ptr if need else None, workspace_bytes=need)
        harness.synchronize()
        raw = np.concatenate([content(hc, nbytes, shift * size), np.frombuffer(stored.tobytes()[nbytes:], np.uint8)])
        got = raw.copy().view(np.float32 if out == "f32" else np.uint16).reshape(m, ldc)
        assert np.array_equal(got[:, n:], stored[:, n:])
        assert first is None or got.tobytes() == first.tobytes()
        first = got
    got = got[:, :n]
    return (got.astype(np.float64) if out == "f32" else to.half_values(got, out)), before[:, :n].astype(np.float64)


def rounded(want, out):
    return want if out == "f32" else to.half_values(to.half_bits(want.astype(np.float32), out), out)


def exactly(m, n, k, fa, fb, blocks, out, accumulate, case, workspace=True, wide=True):
    rng = np.random.default_rng(100 + case)
    ha, hb = operand(fa, m, k, blocks[0], rng), operand(fb, n, k, blocks[1], rng)
    a, b = Matrix(fa, m, k, blocks[0], held=ha, wider=case % 3 if wide else 0), Matrix(fb, n, k, blocks[1], held=hb, wider=case % 2 if wide else 0)
    va, vb = fo.values(*ha, fa, k, blocks[0]).astype(np.float32), fo.values(*hb, fb, k, blocks[1]).astype(np.float32)
    assert np.abs(va).sum(1).max() * np.abs(vb).max() + 64 < 2.0 ** 24, "partial sums are whole numbers that 24 bits hold"
    got, before = product(a, b, out, accumulate, (case % 3) * 5 if wide else 0, case % 4 if wide else 0, workspace, seed_c=case)
    want = (va @ vb.T).astype(np.float64)               # exact in f32
    assert np.array_equal(got, rounded(want + before if accumulate else want, out))


SHAPES = [(1, 1, 1), (1, 16, 32), (1, 64, 128), (1, 65, 4096), (1, 1000, 4128), (2, 33, 100), (3, 128, 256), (7, 260, 513), (8, 300, 640), (15, 64, 1000), (16, 48, 2048), (17, 130, 129), (31, 257, 384),
          (32, 96, 4100), (33, 512, 512), (48, 100, 300), (63, 65, 1025), (64, 64, 64), (65, 1, 300), (100, 100, 100), (128, 128, 256), (129, 127, 255), (200, 768, 768), (256, 256, 512), (257, 255, 2049),
          (300, 1000, 1300), (1000, 257, 256), (513, 514, 515), (96, 2304, 8190), (640, 640, 384), (1030, 1040, 640), (768, 96, 6000), (1, 4096, 16384), (4097, 3, 40), (1, 17, 1024), (3, 100, 1025), (9, 31, 2500),
          (16, 200, 4096), (16, 33, 4097), (2, 1000, 12300), (13, 64, 16640), (5, 70, 17000)]


@pytest.mark.parametrize("out,accumulate", [("bf16", False), ("f32", False), ("f32", True), ("bf16", True), ("f16", False), ("f16", True)])
def test_products_are_exact(out, accumulate):
    for case, (m, n, k) in enumerate(SHAPES):
        fa, fb = [(fo.E4M3, fo.E4M3), (fo.E5M2, fo.E4M3), (fo.E4M3, fo.E5M2), (fo.E5M2, fo.E5M2)][case % 4]
        blocks = [(1, 128), (1, 1), (128, 1), (128, 128)][case // 2 % 4]
        print(f"product {m} x {n} x {k} {out} accumulate {accumulate} formats {fa} {fb} blocks {blocks}", flush=True)
        exactly(m, n, k, fa, fb, blocks, out, accumulate, case)


# a shape of whole tiles and one of ragged ones for every form (the names are those of the table in csrc/f8_forms.hpp; tests/test_host_f8_forms.py asks it)
FORMS = {"256x256": [(3328, 3328, 1024), (3300, 3400, 1000)], "256x128": [(2048, 2560, 1024), (2000, 2300, 1000)], "128x128": [(2048, 2048, 512), (2000, 2050, 500)], "64x64": [(1024, 1024, 512), (500, 1030, 300)]}


@pytest.mark.parametrize("blocks", [(1, 128), (1, 1)])
@pytest.mark.parametrize("out,accumulate", [("bf16", False), ("f32", True)])
@pytest.mark.parametrize("form", list(FORMS))
def test_every_form(form, out, accumulate, blocks):
    for case, (m, n, k) in enumerate(FORMS[form]):
        print(f"form {form}: {m} x {n} x {k} {out} accumulate {accumulate} blocks {blocks}", flush=True)
        exactly(m, n, k, fo.E4M3 if case else fo.E5M2, fo.E4M3, blocks, out, accumulate, case, workspace=False, wide=False)


PARTS = [(17, 64, 16384), (64, 512, 16384), (25, 70, 17000), (130, 100, 20000), (30, 1001, 16000)]


@pytest.mark.parametrize("out,accumulate", [("bf16", True), ("f32", False)])
@pytest.mark.parametrize("m,n,k", PARTS)
def test_parts_of_a_long_axis(m, n, k, out, accumulate):
    print(f"product {m} x {n} x {k} in parts", flush=True)
    assert B.f8_gemm_workspace(m, n, k) > 0
    exactly(m, n, k, fo.E4M3, fo.E4M3, (1, 128), out, accumulate, 7)


@pytest.mark.parametrize("m", [1, 9, 40, 300])
@pytest.mark.parametrize("fa", ["e4m3", "e5m2"])
def test_real_data(fa, m):
    """Any scales, any codes: within the bound of f32 sums, and half a step of the result."""
    rng = np.random.default_rng(m)
    n, k = 200, 1500
    for block_rows in (1, 128):
        ha = fo.quantize((rng.standard_normal((m, k)) * np.exp2(3 * rng.standard_normal((m, 1)))).astype(np.float32), FORMATS[fa])
        hb = fo.quantize((0.02 * rng.standard_normal((n, k))).astype(np.float32), fo.E4M3, block_rows)
        a, b = Matrix(FORMATS[fa], m, k, held=ha), Matrix(fo.E4M3, n, k, block_rows, held=hb)
        va, vb = fo.values(*ha, FORMATS[fa], k), fo.values(*hb, fo.E4M3, k, block_rows)
        want, error = va @ vb.T, fo.sum_error(va, vb)
        for out, half in (("f32", 2.0 ** -24), ("bf16", 2.0 ** -8), ("f16", 2.0 ** -11)):
            got, _ = product(a, b, out)
            if m > 16 and out != "f32":        # seven of eight products cut at 2^-13 of the largest, which is less than 2^-10 of the sum of magnitudes
                error = fo.sum_error(va, vb) + 2.0 ** -10 * (np.abs(va) @ np.abs(vb).T)
            assert np.all(np.abs(got - want) <= error + half * (np.abs(want) + error) + 2.0 ** -25)      # f16 has subnormal numbers of 2^-24


def test_nan_stays_in_its_row_and_column():
    rng = np.random.default_rng(9)
    for m, n, k in [(3, 40, 300), (150, 200, 300)]:
        ha, hb = operand(fo.E4M3, m, k, 1, rng), operand(fo.E4M3, n, k, 1, rng)
        ha[1][1, 2], hb[1][2, 17] = np.nan, np.nan
        a, b = Matrix(fo.E4M3, m, k, held=ha), Matrix(fo.E4M3, n, k, held=hb)
        got, _ = product(a, b, "f32")
        assert np.array_equal(np.isnan(got), (np.arange(m) == 2)[:, None] | (np.arange(n) == 17)[None, :])


def test_nothing_to_contract_over():
    a, b = Matrix(fo.E4M3, 20, 0), Matrix(fo.E4M3, 30, 0)
    got, _ = product(a, b, "f32")
    assert not got.any()
    got, before = product(a, b, "f32", accumulate=True)
    assert np.array_equal(got, before)
    product(Matrix(fo.E4M3, 1, 0), b, "bf16")


def test_offsets_beyond_32_bits():
    """C of 70,000 x 70,000 bf16 is 9.8 GB; A and B are zero but for their last rows, and C is read where those meet."""
    print("product with 9.8 GB of C", flush=True)
    m, k = 70000, 128
    codes = np.zeros((m, k), np.uint8)
    codes[-3:] = fo.nearest_codes(np.arange(1.0, 4.0)[:, None] * np.ones((1, k)), fo.E4M3)
    a = Matrix(fo.E4M3, m, k, held=(codes, np.ones((1, m), np.float32)))
    c = harness.DevBuf(2 * m * m)
    B.proxy_device_fill_async(c.ptr, 0xEE, c.nbytes, 0)
    B.f8_gemm(a.matrix, a.matrix, c.ptr, B.CKPT_BF16, m, 0)
    harness.synchronize()
    for row, want in ((m - 3, 1.0), (m - 1, 3.0), (m // 2, 0.0), (0, 0.0)):
        got = to.half_values(gu.download(c, 2 * (row * m + m - 5), 10).view(np.uint16), "bf16")
        assert np.array_equal(got, 128 * want * np.array([0.0, 0, 1, 2, 3]))
