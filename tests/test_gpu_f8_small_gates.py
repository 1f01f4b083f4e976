"""Gates far below zero beside an `up` so large that the block's value is no small one: act(g) keeps f32's relative accuracy as long as the factor of g is a normal number of f32, and is zero, or nearly right, below."""
import numpy as np
import pytest

from oracle import f8_oracle as fo
from tests.test_gpu_f8_gated import Given, run_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,lowest", [("silu", -96.0), ("gelu", -11.0)])
def test_far_below_zero(name, lowest):
    t, f, d = 130, 256, 128
    g = np.tile(np.linspace(lowest, -0.5, f).astype(np.float32), (t, 1))
    gate, up = Given(g), Given(np.full((t, f), 2.0 ** 100, np.float32))
    dy, wd = Given(np.full((t, d), 2.0 ** 50, np.float32)), Given(np.full((f, d), 2.0 ** 43, np.float32), fo.E4M3, 128)
    out = run_backward(dy, wd, gate.on, up.on, name, (fo.E4M3, fo.E4M3))
    want = fo.backward(dy.v, wd.v, gate.v, up.v, name)
    _, _, z, _ = fo.gate(name, gate.v)
    normal = z[0] > np.log(2.0 ** -126)
    assert 3 < np.sum(~normal) and np.sum(normal) > 200
    for k, of in (("h_by_col", "h"), ("dup_by_col", "dup")):          # a column has one gate: a block's largest value is as small as its others
        value, error = want[of]
        codes, scales = out[k].read()
        assert fo.wrong_rounding(codes[normal], scales[:, normal], value.T[normal], error.T[normal], fo.E4M3) is None, k
        got = fo.values(codes, scales, fo.E4M3, t)[~normal]
        assert np.all(np.abs(got) <= 1.07 * np.abs(value.T[~normal]))          # half a step is 2^-4, and f32 errors
