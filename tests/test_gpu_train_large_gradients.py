"""A step that is given the norm leaves no moment infinite or NaN: gradients whose squares f32 does not hold are flagged as infinities are, and change nothing, unless the clipping brings them
down. The limit is 2^63 for scale * norm: squares up to 2^126 have room for rounding up in 8 bits."""
import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2406_10707_amd import binding as B
from paper_2406_10707_amd import harness
from tests import gpu_util as gu
from tests.test_gpu_train_optim import Arena

pytestmark = pytest.mark.gpu

N = 333


class Step:
    def __init__(self, grad, bits, values):
        self.bits, self.norm = bits, harness.DevBuf(24)
        rng = np.random.default_rng(3)
        g = (1e-3 * rng.standard_normal(N)).astype(np.float32)
        g[40:40 + len(values)] = values
        self.arena = Arena(N * 20 + 8192)
        add = self.arena.add
        self.g = g if grad == "f32" else to.half_values(to.half_bits(g, "bf16"), "bf16").astype(np.float32)
        t = dict(numel=N, weight_decay=0.1, grad=add(g if grad == "f32" else to.half_bits(g, "bf16"), 4, 0), master=add((0.02 * rng.standard_normal(N)).astype(np.float32), 4, 0),
                 param=add(np.zeros(N, np.uint16), 2, 0))
        if bits == 32:
            t |= dict(m=add(np.full(N, 1e-3, np.float32), 4, 0), v=add(np.full(N, 1e-6, np.float32), 4, 0))
        else:
            t |= dict(m=add(np.full(N, 0x38, np.uint8), 1, 0), v=add(np.full(N, 0x38, np.uint8), 1, 0), m_scale=add(np.full(11, 117, np.uint8), 1, 0), v_scale=add(np.full(11, 107, np.uint8), 1, 0))
        self.arena.upload()
        self.before = gu.download(self.arena.buf)
        self.opt = B.Optimizer([t], grad_dtype=B.CKPT_F32 if grad == "f32" else B.CKPT_BF16, state_bits=bits)

    def run(self, max_norm, grad_scale=1.0):
        """The norm's result; two steps are made, so that what the first has left in the moments counts."""
        self.opt.grad_norm(self.norm.ptr, 0, max_norm=max_norm, grad_scale=grad_scale)
        for n in (1, 2):
            self.opt.step(0, step=n, lr=1e-3, beta1=0.0, beta2=0.0, seed=n, stochastic=True, norm=self.norm.ptr)
        harness.synchronize()
        return B.ckpt_norm_result.from_buffer_copy(gu.download(self.norm).tobytes())

    def changed(self):
        return not np.array_equal(self.before, gu.download(self.arena.buf))

    def whole(self):
        """Weights and moments are finite."""
        self.arena.fetch()
        w = self.arena.read(1).view(np.float32)
        if self.bits == 32:
            return all(np.isfinite(x).all() for x in (w, self.arena.read(3).view(np.float32), self.arena.read(4).view(np.float32)))
        return np.isfinite(w).all() and all((self.arena.read(k) != 255).all() for k in (5, 6))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("values,max_norm,grad_scale", [([2e19], 0.0, 1.0), ([-1e30], 0.0, 1.0), ([2e19], 1e25, 1.0), ([2e9], 0.0, 1e10), ([2.0 ** 63 * 1.015625], 0.0, 1.0),
                                                         ([3e38] * 4, 1.0, 1.0), ([np.inf], 1.0, 1.0), ([np.nan], 0.0, 1.0)])
def test_what_f32_does_not_hold_is_left_out(values, max_norm, grad_scale, grad, bits):
    print(f"gradients {values} {grad}, max_norm {max_norm:g}, grad_scale {grad_scale:g}, {bits} bits", flush=True)
    s = Step(grad, bits, values)
    r = s.run(max_norm, grad_scale)
    assert r.nonfinite == 1 and r.scale == 0 and not s.changed()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("values,max_norm,grad_scale", [([2e19], 1.0, 1.0), ([1e36, -1e36], 1.0, 1.0), ([1e30], 0.0, 1e-20), ([2.0 ** 63], 0.0, 1.0), ([2.0 ** 100], 2.0 ** 62, 1.0)])
def test_what_it_holds_is_not(values, max_norm, grad_scale, grad, bits):
    print(f"gradients {values} {grad}, max_norm {max_norm:g}, grad_scale {grad_scale:g}, {bits} bits", flush=True)
    s = Step(grad, bits, values)
    norm = float(np.sqrt(np.sum(s.g.astype(np.float64) ** 2))) * grad_scale
    r = s.run(max_norm, grad_scale)
    want = grad_scale * (max_norm / norm if 0 < max_norm < norm else 1.0)
    assert r.nonfinite == 0 and abs(r.scale - want) <= 2.0 ** -23 * want and abs(r.norm - norm) <= 2.0 ** -23 * norm
    assert s.changed() and s.whole()
