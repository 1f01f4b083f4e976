"""The oracle of the 8-bit operators against independent statements: format tables and rounding against torch's float8 types, slopes against differences."""
import numpy as np
import pytest

from oracle import f8_oracle as fo

torch = pytest.importorskip("torch")
TYPES = {fo.E4M3: torch.float8_e4m3fn, fo.E5M2: torch.float8_e5m2}


@pytest.mark.parametrize("fmt", [fo.E4M3, fo.E5M2])
def test_every_code(fmt):
    want = torch.arange(256, dtype=torch.uint8).view(TYPES[fmt]).double().numpy()
    assert np.array_equal(fo.TABLE[fmt], want, equal_nan=True)


@pytest.mark.parametrize("fmt", [fo.E4M3, fo.E5M2])
def test_rounding(fmt):
    rng = np.random.default_rng(1)
    finite = np.sort(np.abs(fo.TABLE[fmt][np.isfinite(fo.TABLE[fmt])]))
    y = np.concatenate([finite, (finite[1:] + finite[:-1]) / 2, np.nextafter(np.float32((finite[1:] + finite[:-1]) / 2), np.float32(0)).astype(np.float64), rng.random(10000) * finite[-1], 2.0 ** rng.uniform(-30, 8, 10000)])
    y = np.concatenate([y, -y]).astype(np.float32)
    assert np.array_equal(fo.nearest_codes(y, fmt), torch.from_numpy(y).to(TYPES[fmt]).view(torch.uint8).numpy())


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fmt", [fo.E4M3, fo.E5M2])
def test_blocks(fmt, block_rows):
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((200, 300)) * 2.0 ** rng.integers(-20, 20, (200, 1))).astype(np.float32)
    x[5, 128:256] = 0
    codes, scales = fo.quantize(x, fmt, block_rows)
    assert codes.shape == (200, 384) and scales.shape == (3, -(-200 // block_rows)) and not codes[:, 300:].any()
    v = fo.values(codes, scales, fmt, 300, block_rows)
    for r in range(0, 200, block_rows):
        for c in range(0, 300, 128):
            block, got = x[r:r + block_rows, c:c + 128].astype(np.float64), v[r:r + block_rows, c:c + 128]
            scale = max(np.abs(block).max() / fo.MOST[fmt], 2.0 ** -126)
            assert abs(scales[c // 128, r // block_rows] - scale) <= scale * 2.0 ** -24
            assert np.all(np.abs(got - block) <= np.maximum(fo.HALF_STEP[fmt] * np.abs(block), fo.HALF_SMALLEST[fmt] * scale) * (1 + 2.0 ** -20))
    x[3, 7] = np.inf
    x[180, 290] = np.nan
    bad = np.isnan(fo.quantize(x, fmt, block_rows)[1])
    assert bad[0, 3 // block_rows] and bad[2, 180 // block_rows] and bad.sum() == 2


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_slopes_against_differences(name):
    g = np.linspace(-12, 12, 2001)
    d = 1e-5
    numeric = (fo.gate(name, g + d)[0] - fo.gate(name, g - d)[0]) / (2 * d)      # off by d^2 / 6 of a third derivative below 3, and 2^-52 * 12 / d
    assert np.max(np.abs(numeric - fo.gate(name, g)[1])) < 1e-9
    t = torch.from_numpy(g)
    want = torch.nn.functional.silu(t) if name == "silu" else torch.nn.functional.gelu(t, approximate="tanh")
    assert np.allclose(fo.gate(name, g)[0], want.numpy(), rtol=1e-13, atol=1e-15)


@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gradients_of_the_block_against_differences(name):
    """d(sum(dy * y)) / d(every input) of y = (act(x Wg^T) * (x Wu^T)) Wd^T, by the formulas and by central differences."""
    rng = np.random.default_rng(3)
    x, wg, wu, wd, dy = (rng.standard_normal(s) for s in ((5, 6), (7, 6), (7, 6), (4, 7), (5, 4)))

    def loss(x, wg, wu, wd):
        return np.sum(dy * ((fo.gate(name, x @ wg.T)[0] * (x @ wu.T)) @ wd.T))
    made = fo.backward(dy, wd.T, x @ wg.T, x @ wu.T, name)
    dgate, dup, h = (made[k][0] for k in ("dgate", "dup", "h"))
    formula = {"x": dgate @ wg + dup @ wu, "wg": dgate.T @ x, "wu": dup.T @ x, "wd": dy.T @ h}
    inputs = {"x": x, "wg": wg, "wu": wu, "wd": wd}
    for which, v in inputs.items():
        for at in np.ndindex(*v.shape):
            step = np.zeros_like(v)
            step[at] = 1e-5
            numeric = (loss(**{**inputs, which: v + step}) - loss(**{**inputs, which: v - step})) / 2e-5
            assert abs(numeric - formula[which][at]) < 1e-7
