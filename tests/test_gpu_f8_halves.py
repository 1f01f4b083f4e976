"""The gated block's forward pass where the tiles of the last round go in halves: both activations, both formats of x, both kinds of blocks, kept or not, last tiles whose second half holds no token. (tests/test_host_f8_halves.py asks whether
these sizes take that way.)"""
import pytest

from oracle import f8_oracle as fo
from tests.test_gpu_f8_gated import check_forward

pytestmark = pytest.mark.gpu

HALVES = [(4000, 200, 2100), (3900, 129, 2176), (4096, 384, 2050)]


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fx", [fo.E4M3, fo.E5M2])
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_halves(name, fx, block_rows):
    for case, (t, d, f) in enumerate(HALVES):
        check_forward(t, d, f, name, (case + block_rows) % 2 == 0, fx, fo.E4M3, block_rows, case)
