"""The product of two MXFP4 matrices. Values and scales are chosen so that every partial sum is a multiple of the smallest product that
24 bits hold: f32 sums are then exact in any order, and the result is compared bit for bit. One test with real data has the bound
that f32 accumulation gives."""
import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu
from tests.test_gpu_train_mx import content, guarded

pytestmark = pytest.mark.gpu


def operand(rows, k, rng, spread):
    """(codes, scale bytes) with scales 2^0 .. 2^spread."""
    codes = rng.integers(0, 16, (rows, k)).astype(np.uint8)
    return codes, (127 + rng.integers(0, spread + 1, (rows, -(-k // 32)))).astype(np.uint8)


def on_device(codes, byte):
    cp, sp = B.mx_layout(to.MXFP4, *codes.shape)
    c, s = to.pack_rows(codes, byte, to.MXFP4, cp, sp)
    held = guarded(c.size, c.tobytes()) + guarded(s.size, s.tobytes())
    return held, B.mx_matrix(to.MXFP4, codes.shape[0], codes.shape[1], held[1], cp, held[3], sp)


def product(a, b, m, n, k, out, accumulate, pad, rng, workspace=True, shift=0):
    """(result, C before) as float64."""
    ha, ma = on_device(*a)
    hb, mb = on_device(*b)
    size = 4 if out == "f32" else 2
    ldc = n + pad
    before = rng.integers(-64, 65, (m, ldc)).astype(np.float32)
    stored = before if out == "f32" else to.half_bits(before, "bf16")
    nbytes = (m * ldc - pad) * size
    hc, cptr = guarded(nbytes, stored.tobytes()[:nbytes], shift * size)
    ws_bytes = B.mx_gemm_workspace(m, n, k) if workspace else 0
    ws = harness.DevBuf(max(ws_bytes, 16))
    ws.upload(np.full(ws.nbytes, 0xFF, np.uint8))       # its contents do not matter
    for again in range(2):
        B.proxy_copy_h2d(cptr, stored.ctypes.data, nbytes)
        B.mx_gemm(ma, mb, cptr, B.CKPT_F32 if out == "f32" else B.CKPT_BF16, ldc, 0, accumulate=accumulate, workspace=ws.ptr if ws_bytes else None, workspace_bytes=ws_bytes)
        harness.synchronize()
        raw = np.concatenate([content(hc, nbytes, shift * size), stored.tobytes()[nbytes:] and np.frombuffer(stored.tobytes()[nbytes:], np.uint8)]
                             if pad else [content(hc, nbytes, shift * size)])
        got = raw.copy().view(np.float32 if out == "f32" else np.uint16).reshape(m, ldc)
        assert np.array_equal(got[:, n:], stored[:, n:])
        if again:
            assert got.tobytes() == first.tobytes()
        first = got
    got = got[:, :n]
    return (got.astype(np.float64) if out == "f32" else to.half_values(got, "bf16")), before[:, :n].astype(np.float64)


def exactly(want, out):
    return want if out == "f32" else to.half_values(to.half_bits(want.astype(np.float32), "bf16"), "bf16")


SHAPES = [(1, 1, 1), (1, 16, 32), (1, 64, 128), (1, 65, 4096), (1, 1000, 4128), (2, 33, 100), (3, 128, 256), (7, 260, 513), (8, 300, 640), (15, 64, 1000), (16, 48, 2048), (17, 130, 129),
          (31, 257, 384), (32, 96, 4100), (33, 512, 512), (48, 100, 300), (63, 65, 1025), (64, 64, 64), (65, 1, 300), (100, 100, 100), (128, 128, 256), (129, 127, 255),
          (200, 768, 768), (256, 256, 512), (257, 255, 2049), (300, 1000, 1300), (1000, 257, 256), (513, 514, 515), (96, 2304, 8190), (640, 640, 384), (1030, 1040, 640),
          (768, 96, 6000), (1, 4096, 16384), (4097, 3, 40),
          (1, 17, 1024), (3, 100, 1025), (9, 31, 2500), (16, 200, 4096), (16, 33, 4097), (2, 1000, 12300), (13, 64, 16640), (5, 70, 17000)]


@pytest.mark.parametrize("out,accumulate", [("bf16", False), ("f32", False), ("f32", True), ("bf16", True)])
def test_products_are_exact(out, accumulate):
    for k, (m, n, kk) in enumerate(SHAPES):
        print(f"product {m} x {n} x {kk} {out} accumulate {accumulate}", flush=True)
        rng = np.random.default_rng(50 + k)
        a, b = operand(m, kk, rng, 1), operand(n, kk, rng, 1)
        want, magnitude = to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))
        assert magnitude.max() + 64 < 2.0 ** 22, "partial sums are multiples of 1/4 that 24 bits hold"
        got, before = product(a, b, m, n, kk, out, accumulate, (k % 3) * 5, rng, shift=k % 4)
        assert np.array_equal(got, exactly(want + before if accumulate else want, out))


# a shape of whole tiles and one of ragged ones for every form (the names are those of the table in csrc/mx_gemm_forms.hpp; tests/test_host_train_forms.py asks it)
FORMS = {"256x256": [(3328, 3328, 1024), (3300, 3400, 1000)], "192x192": [(2496, 3264, 2048), (2500, 3300, 2000)], "128x128": [(2048, 2048, 2048), (2000, 2050, 1030)],
         "64x128": [(2048, 2048, 1024), (2040, 1950, 1000)], "64x64 four stages": [(1024, 1024, 1024), (500, 1030, 2000)], "64x64 two stages": [(1024, 2304, 768), (1000, 2300, 700)]}


@pytest.mark.parametrize("out,accumulate", [("bf16", False), ("f32", True), ("bf16", True), ("f32", False)])
@pytest.mark.parametrize("form", list(FORMS))
def test_every_form(form, out, accumulate):
    for m, n, k in FORMS[form]:
        print(f"form {form}: {m} x {n} x {k} {out} accumulate {accumulate}", flush=True)
        rng = np.random.default_rng(m + n)
        a, b = operand(m, k, rng, 0), operand(n, k, rng, 0)
        want, magnitude = to.gemm(to.values(*a, to.MXFP4).astype(np.float32), to.values(*b, to.MXFP4).astype(np.float32))      # exact in f32 as well
        assert magnitude.max() + 64 < 2.0 ** 22
        got, before = product(a, b, m, n, k, out, accumulate, 0, rng, workspace=False)
        assert np.array_equal(got, exactly(want.astype(np.float64) + before if accumulate else want, out))


@pytest.mark.parametrize("out,accumulate", [("bf16", True), ("f32", False)])
@pytest.mark.parametrize("m,n,k", [(17, 64, 16384), (64, 512, 16384), (25, 70, 17000), (130, 100, 20000), (30, 1001, 16000)])
def test_parts_of_a_long_axis(m, n, k, out, accumulate):
    print(f"product {m} x {n} x {k} in parts", flush=True)
    assert B.mx_gemm_workspace(m, n, k) > 0
    rng = np.random.default_rng(6)
    a, b = operand(m, k, rng, 0), operand(n, k, rng, 0)
    want, magnitude = to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))
    assert magnitude.max() + 64 < 2.0 ** 22
    got, before = product(a, b, m, n, k, out, accumulate, 3, rng, shift=1)
    assert np.array_equal(got, exactly(want + before if accumulate else want, out))


def test_offsets_beyond_32_bits():
    """C of 70,000 x 70,000 bf16 is 9.8 GB; A and B are zero but for their last rows, and C is read where those meet."""
    print("product with 9.8 GB of C", flush=True)
    n, k, tail = 70000, 256, 48
    rng = np.random.default_rng(8)
    a, b = operand(tail, k, rng, 0), operand(tail, k, rng, 0)
    mats, held = [], []
    for codes, byte in (a, b):
        cp, sp = B.mx_layout(to.MXFP4, n, k)
        pc, ps = to.pack_rows(codes, byte, to.MXFP4, cp, sp)
        c, s = harness.DevBuf(n * cp), harness.DevBuf(n * sp)
        held += [c, s]
        for buf, part, pitch in ((c, pc, cp), (s, ps, sp)):
            B.proxy_device_fill_async(buf.ptr, 0, buf.nbytes, 0)
            B.proxy_copy_h2d(buf.ptr + (n - tail) * pitch, part.ctypes.data, part.nbytes)
        mats.append(B.mx_matrix(to.MXFP4, n, k, c.ptr, cp, s.ptr, sp))
    c = harness.DevBuf(2 * n * n)
    B.proxy_device_fill_async(c.ptr, 0xEE, c.nbytes, 0)
    B.mx_gemm(mats[0], mats[1], c.ptr, B.CKPT_BF16, n, 0)
    harness.synchronize()
    want = exactly(to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))[0], "bf16")
    for i in range(tail):
        row = to.half_values(gu.download(c, 2 * ((n - tail + i) * n), 2 * n).view(np.uint16), "bf16")
        assert np.array_equal(row[n - tail:], want[i]) and not row[: n - tail].any()
    for row in (0, 33333, n - tail - 1):
        assert not to.half_values(gu.download(c, 2 * row * n, 2 * n).view(np.uint16), "bf16").any()
    for buf in held + [c]:
        buf.free()


@pytest.mark.parametrize("m,n,k", [(1, 64, 16384), (96, 96, 8192), (64, 200, 5000)])
def test_without_workspace(m, n, k):
    print(f"product {m} x {n} x {k} without workspace", flush=True)
    rng = np.random.default_rng(3)
    a, b = operand(m, k, rng, 0), operand(n, k, rng, 0)
    want, _ = to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))
    got, _ = product(a, b, m, n, k, "f32", False, 0, rng, workspace=False)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("m,n,k", [(1, 512, 4096), (40, 300, 1000), (300, 300, 2000), (520, 1030, 1024)])
def test_real_data_within_the_bound_of_f32_sums(m, n, k):
    """K additions, each off by at most 2^-23 of the magnitudes' sum (rounding towards zero allowed for)."""
    print(f"product of real data {m} x {n} x {k}", flush=True)
    rng = np.random.default_rng(4)
    a = to.quantize(rng.standard_normal((m, k)).astype(np.float32), to.MXFP4)
    b = to.quantize((rng.standard_normal((n, k)) * 2.0 ** rng.integers(-12, 3, (n, k))).astype(np.float32), to.MXFP4)
    want, magnitude = to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))
    got, _ = product(a, b, m, n, k, "f32", False, 0, rng)
    assert np.all(np.abs(got - want) <= k * 2.0 ** -23 * magnitude)


@pytest.mark.parametrize("m,n,k", [(1, 70, 600), (20, 64, 256), (70, 130, 700), (300, 520, 1024)])
def test_nan_scales_reach_their_row_or_column_alone(m, n, k):
    print(f"product with NaN {m} x {n} x {k}", flush=True)
    rng = np.random.default_rng(5)
    a, b = operand(m, k, rng, 0), operand(n, k, rng, 0)
    a[1][m // 2, -1] = 255
    b[1][n - 1, 0] = 255
    want, _ = to.gemm(to.values(*a, to.MXFP4), to.values(*b, to.MXFP4))
    got, _ = product(a, b, m, n, k, "f32", False, 0, rng)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
    assert np.isnan(want).sum() == m + n - 1


@pytest.mark.parametrize("accumulate", [False, True])
def test_no_columns_give_zeros(accumulate):
    print("K = 0", flush=True)
    c, ptr = guarded(3 * 5 * 4, np.full(15, 7, np.float32).tobytes())
    a, b = (B.mx_matrix(B.CKPT_MXFP4, r, 0, None, 0, None, 0) for r in (3, 5))
    B.mx_gemm(a, b, ptr, B.CKPT_F32, 5, 0, accumulate=accumulate)
    harness.synchronize()
    assert np.all(content(c, 60).copy().view(np.float32) == (7 if accumulate else 0))


def test_what_is_refused():
    print("refusals", flush=True)
    buf, small = harness.DevBuf(1 << 20), harness.DevBuf(1024)
    c = buf.ptr + (512 << 10)
    good = dict(fmt=B.CKPT_MXFP4, rows=64, cols=256, codes=buf.ptr, code_pitch=128, scales=buf.ptr + 65536, scale_pitch=16)

    def refused(text, c=c, dtype=B.CKPT_F32, ldc=64, code=B.CKPT_EINVAL, b=None, **change):
        with pytest.raises(B.CkptError) as e:
            B.mx_gemm(B.mx_matrix(**{**good, **change}), B.mx_matrix(**{**good, **(b or {})}), c, dtype, ldc, 0)
        assert e.value.code == code and text in e.value.text, e.value.text

    refused("CKPT_MXFP4", fmt=B.CKPT_MXFP8)
    refused("columns", cols=250)
    refused("c_dtype", dtype=B.CKPT_F16)
    refused("ldc", ldc=63)
    refused("aligned", c=c + 2)
    refused("C: null", c=None)
    refused("C: range runs past", c=small.ptr)
    refused("A: range runs past", rows=1 << 20)
    refused("B: pitches", b=dict(scale_pitch=24))
    refused("B: null", b=dict(scales=None))
    harness.synchronize()
