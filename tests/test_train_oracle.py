"""The oracle of the training operators against what can be said without it: the formats' definitions bit by bit, rounding by brute
force, the mean of stochastic rounding; and the header against the binding."""
import os
import re

import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ckpt_train.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(ckpt_[a-z0-9_]+)\s*\(", text))
    assert declared == set(B.EXPORTED_TRAIN)
    for name in declared:
        assert hasattr(B.lib, name)


def test_the_tables_are_the_formats():
    for code in range(8):
        e, m = code >> 1, code & 1
        assert to.FP4[code] == (m * 0.5 if e == 0 else 2.0 ** (e - 1) * (1 + m / 2))
    for code in range(127):
        e, m = code >> 3, code & 7
        assert to.FP8[code] == (m / 8 * 2.0 ** -6 if e == 0 else 2.0 ** (e - 7) * (1 + m / 8))
    assert to.FP8[-1] == 448


@pytest.mark.parametrize("fmt", [to.MXFP4, to.MXFP8])
def test_nearest_is_nearest_with_ties_to_even_codes(fmt):
    grid = to.GRID[fmt]
    mid = (grid[1:] + grid[:-1]) / 2
    y = np.concatenate([grid, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9)])
    y = np.concatenate([y, -y])
    got = to.element_codes(y, fmt)
    for value, code in zip(y, got):
        far = np.abs(grid - abs(value))
        best = np.flatnonzero(far == far.min())
        want = best[0] if len(best) == 1 else best[best % 2 == 0][0]
        assert code == want + (to.SIGN[fmt] if np.signbit(value) else 0)


@pytest.mark.parametrize("fmt", [to.MXFP4, to.MXFP8])
def test_scales_are_the_smallest_that_fit(fmt):
    rng = np.random.default_rng(1)
    top = to.GRID[fmt][-1]
    peaks = np.concatenate([top * 2.0 ** np.arange(-20, 20), np.exp(rng.uniform(-60, 60, 500))]).astype(np.float32).astype(np.float64)
    peaks = np.concatenate([peaks, np.nextafter(peaks.astype(np.float32), np.float32(1e38)).astype(np.float64)])
    blocks = np.zeros((len(peaks), 32))
    blocks[:, 5] = -peaks
    e = to.scale_bytes(blocks, fmt).astype(np.float64) - 127
    assert np.all(peaks <= top * 2.0 ** e) and np.all(peaks > top * 2.0 ** (e - 1))
    assert to.scale_bytes(np.zeros((1, 32)), fmt)[0] == 0
    for bad in (np.inf, -np.inf, np.nan):
        blocks[0, 3] = bad
        assert to.scale_bytes(blocks, fmt)[0] == 255


@pytest.mark.parametrize("fmt", [to.MXFP4, to.MXFP8])
def test_stochastic_rounding_has_the_value_as_its_mean(fmt):
    grid = to.GRID[fmt]
    random = np.arange(65536)
    for y in (grid[1] / 3, grid[-1] * 0.9, grid[-2], 1.3, -0.7):
        v = to.values(to.element_codes(np.full(65536, y), fmt, random).reshape(1, -1), np.full((1, 2048), 127, np.uint8), fmt)
        step = np.max(np.diff(grid))
        assert abs(v.mean() - y) <= step / 65536 and set(np.unique(np.abs(v))) <= set(grid)


def test_rows_draw_random_numbers_of_their_own():
    a = to.bits16(7, 3, 6)
    assert np.array_equal(a.reshape(-1)[:6], to.bits16(7, 1, 6)[0]) and np.array_equal(a[1], to.bits16(9, 1, 6)[0])
    assert a.min() >= 0 and a.max() < 65536


def test_an_unknown_field_of_a_tensor_is_refused():
    """A misspelt weight_decay would otherwise be 0."""
    for tensor in (dict(numel=4, grad=0, weight_deacy=0.1), dict(numel=4, dev_grad=0)):
        with pytest.raises(TypeError, match="weight_deacy|dev_grad"):
            B.Optimizer([tensor])
