"""The workspace of the 8-bit operators: just the bytes that a call asked for, between guards and full of NaN. Nothing behind them is written, nothing is read that the call has not written; with fewer bytes the result is as right."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests.f8_device import Matrix
from tests.test_gpu_f8_gated import ACT, Given, rows_of
from tests.test_gpu_f8_gemm import PARTS, operand, rounded
from tests.test_gpu_train_mx import DTYPES, content, guarded

pytestmark = pytest.mark.gpu


def nan_bytes(nbytes):
    return guarded(nbytes, b"\xff" * nbytes)


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,n,k", PARTS)
def test_product(m, n, k, out):
    rng = np.random.default_rng(m)
    ha, hb = operand(fo.E4M3, m, k, 1, rng), operand(fo.E4M3, n, k, 128, rng)
    a, b = Matrix(fo.E4M3, m, k, held=ha), Matrix(fo.E4M3, n, k, 128, held=hb)
    va, vb = fo.values(*ha, fo.E4M3, k), fo.values(*hb, fo.E4M3, k, 128)
    assert np.abs(va).sum(1).max() * np.abs(vb).max() < 2.0 ** 24
    code, size = DTYPES[out]
    need = B.f8_gemm_workspace(m, n, k)
    for given in (need, need // 2 // 16 * 16, 16):
        print(f"product {m} x {n} x {k} {out} with {given} of {need} bytes", flush=True)
        ws, at = nan_bytes(given)
        c, c_at = guarded(m * n * size)
        B.f8_gemm(a.matrix, b.matrix, c_at, code, n, 0, workspace=at, workspace_bytes=given)
        harness.synchronize()
        content(ws, given)
        got = content(c, m * n * size).copy().view(np.float32 if out == "f32" else np.uint16).reshape(m, n)
        assert np.array_equal(got if out == "f32" else to.half_values(got, out), rounded(va @ vb.T, out))


# up to eight and up to sixteen rows; values first; ragged
@pytest.mark.parametrize("t,d,f", [(1, 300, 200), (8, 129, 4097), (3, 4100, 33), (16, 640, 1000), (17, 300, 4090), (64, 129, 4224), (40, 256, 16384)])
@pytest.mark.parametrize("keep", [False, True])
def test_gated_forward(keep, t, d, f):
    rng = np.random.default_rng(t)
    x = Given(rows_of(rng, (t, d)))
    wg, wu = (Given((rng.standard_normal((f, d)) / d ** 0.5).astype(np.float32), fo.E4M3, 128) for _ in range(2))
    want = fo.forward(x.v, wg.v, wu.v, "gelu")
    need = B.gated_workspace(t, f, d)
    assert need > 0
    for given in (need, need - 16):
        print(f"gated {t} x {d} x {f} keep {keep} with {given} of {need} bytes", flush=True)
        ws, at = nan_bytes(given)
        out = {k: Matrix(fo.E4M3, t, f) for k in (("gate", "up", "h") if keep else ("h",))}
        B.gated_forward(x.on.matrix, wg.on.matrix, wu.on.matrix, ACT["gelu"], 0, **{k: m.matrix for k, m in out.items()}, workspace=at, workspace_bytes=given)
        harness.synchronize()
        left = content(ws, given)
        assert given == need or np.all(left == 0xFF)          # too small to be used
        for k, m in out.items():
            assert fo.wrong_rounding(*m.read(), *want[k], fo.E4M3) is None, k
