"""What the sums of 8-bit products keep of small products beside large ones: all of it where they are sums in f32 (C in f32 and f16, and up to sixteen rows of A). Products are whole numbers below 2^24 with large ones that cancel, so that sums in f32 are exact in any order."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from paper_2406_10707_amd import binding as B
from tests.f8_device import FORMATS, Matrix
from tests.test_gpu_f8_gemm import product, rounded

pytestmark = pytest.mark.gpu


def held(v, fmt, block_rows=1, scale=1.0):
    codes = np.zeros((v.shape[0], fo.padded(v.shape[1])), np.uint8)
    codes[:, : v.shape[1]] = fo.nearest_codes(v, fmt)
    assert np.array_equal(fo.TABLE[fmt][codes[:, : v.shape[1]]], v), "values of the format"
    return codes, np.full((codes.shape[1] // 128, -(-v.shape[0] // block_rows)), scale, np.float32)


def multiplied(va, vb, fmt, out, block_rows=1, scale=1.0):
    a, b = Matrix(fmt, *va.shape, held=held(va, fmt, scale=scale)), Matrix(fmt, *vb.shape, block_rows, held=held(vb, fmt, block_rows))
    return product(a, b, out)[0]


def one_large_in_eight(rng, m, n, k):
    """Whole numbers up to 2, but for one 256 in every eight of K, of B and, with signs in turn, of A: 2^16 beside seven products of at most 4. With k a multiple of 16 the large ones of every block of 128 cancel, and any sum of a block's
    products is a whole number below 16 (2^16 + 28) < 2^21."""
    a, b = (rng.choice([-2.0, -1.0, 1.0, 2.0], s) for s in ((m, k), (n, k)))
    at = np.arange(0, k, 8) + rng.integers(0, 8, k // 8)
    a[:, at], b[:, at] = np.where(np.arange(k // 8) % 2, -256.0, 256.0), 256.0
    return a, b


# rows for the kernel of up to sixteen and for tiles; a K that is split among blocks
@pytest.mark.parametrize("m,n,k", [(5, 40, 256), (16, 33, 1040), (17, 40, 256), (40, 33, 1040), (300, 200, 272), (17, 64, 16384)])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("out", ["f32", "f16"])
def test_sums_in_f32_keep_small_products(out, fmt, m, n, k):
    for block_rows in (1, 128):
        print(f"small products beside large ones, {m} x {n} x {k} {fmt} to {out} block_rows {block_rows}", flush=True)
        a, b = one_large_in_eight(np.random.default_rng(m + k), m, n, k)
        assert np.array_equal(multiplied(a, b, FORMATS[fmt], out, block_rows), rounded(a @ b.T, out))


def test_sums_of_f16_are_not_cut():
    """2^16 and seven products of 7 in every eight, nothing cancels: 1024.77, which f16 rounds to 1025; without the small ones it would be 1024."""
    a, b = np.full((40, 128), 3.5), np.full((24, 128), 2.0)
    a[:, ::8] = b[:, ::8] = 256
    got = multiplied(a, b, fo.E4M3, "f16", scale=2.0 ** -10)
    assert np.all(got == 1025) and np.array_equal(got, rounded(a @ b.T / 1024, "f16"))


def test_a_split_product_has_parts_here():
    assert B.f8_gemm_workspace(17, 64, 16384) > 0
