"""What is not zero never becomes zero under CKPT_ROUND_NONZERO, however far below its block's largest value it lies: quantisation and the 8-bit second moment, code by code against the
oracle, which scales in 64 bits."""
import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests.test_gpu_train_mx import quantized_on_device
from tests.test_gpu_train_optim import Arena

pytestmark = pytest.mark.gpu

TINY = [1e-30, 1e-38, 2.0 ** -126, 1e-40, 2.0 ** -149, 1e-10, 1.0]


@pytest.mark.parametrize("rounding", [B.CKPT_ROUND_NONZERO, B.CKPT_ROUND_NONZERO | B.CKPT_ROUND_STOCHASTIC])
@pytest.mark.parametrize("dtype,largest", [("f32", 1e30), ("f32", 3e38), ("f32", 500.0), ("bf16", 1e30), ("f16", 6e4)])
def test_blocks_of_far_magnitudes(dtype, largest, rounding):
    print(f"fp8 nonzero, {dtype} up to {largest:g}, rounding {rounding}", flush=True)
    rng = np.random.default_rng(11)
    rows, cols = 5, 1100
    x = rng.choice([largest, *TINY, 0.0, -0.0], (rows, cols)) * rng.choice([1, -1], (rows, cols))
    x[:, ::32] = largest
    x[2] = rng.choice([*TINY, 0.0], cols)
    stored = x.astype(np.float32) if dtype == "f32" else to.half_bits(x.astype(np.float32), dtype)
    values = stored.astype(np.float64) if dtype == "f32" else to.half_values(stored, dtype)
    _, _, got, _ = quantized_on_device(stored, dtype, rows, cols, cols + 1, 1, to.MXFP8, True, False, rounding, 21)
    key = int(to.mix(np.uint64(21))) if rounding & B.CKPT_ROUND_STOCHASTIC else None
    codes, scales = to.quantize(values, to.MXFP8, key, True)
    assert np.array_equal((codes & 0x7F) == 0, values == 0)
    assert np.array_equal(got[0][1], scales) and np.array_equal(got[0][0], codes)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_second_moments_of_far_gradients(grad, stochastic):
    print(f"8-bit step, gradients from 1e-22 to 1e15, {grad}, stochastic {stochastic}", flush=True)
    rng = np.random.default_rng(12)
    n = 4096 + 77
    g = (rng.choice([1e15, 1e-5, 1e-15, 3e-20, 1e-22, 0.0], n) * rng.standard_normal(n)).astype(np.float32)
    g[::32] = 1e15
    stored = g if grad == "f32" else to.half_bits(g, "bf16")
    if grad == "bf16":
        g = to.half_values(stored, "bf16").astype(np.float32)
    zero = np.zeros(n, np.uint8)
    arena = Arena(n * 20 + 16384)
    t = dict(numel=n, weight_decay=0.0, grad=arena.add(stored, g.itemsize, 0), master=arena.add(np.zeros(n, np.float32), 4, 0))
    first = len(arena.parts)
    t |= dict(m=arena.add(zero, 1, 1), v=arena.add(zero, 1, 2), m_scale=arena.add(zero[: -(-n // 32)], 1, 0), v_scale=arena.add(zero[: -(-n // 32)], 1, 0))
    arena.upload()
    opt = B.Optimizer([t], grad_dtype=B.CKPT_F32 if grad == "f32" else B.CKPT_BF16, param_dtype=0, state_bits=8)
    opt.step(0, step=4, lr=1e-3, beta1=0.9, beta2=0.95, seed=5, stochastic=stochastic)
    harness.synchronize()
    arena.fetch()
    none = np.zeros(n, np.float32)
    m, v = to.moments(none, none, g, 1.0, 0.9, 0.95)
    rm, rv = to.step_bits16(5, 4, 0, n) if stochastic else (None, None)
    assert np.count_nonzero((v > 0) & (v < 1e-30)) > 1000
    for k, (x, r) in enumerate(((m, rm), (v, rv))):
        codes, scales = to.moment8(x, r, nonzero=k == 1)
        assert np.array_equal(arena.read(first + 2 + k), scales) and np.array_equal(arena.read(first + k), codes)
    assert np.all((arena.read(first + 1) > 0) | (v == 0)) and np.isfinite(arena.read(1).view(np.float32)).all()
