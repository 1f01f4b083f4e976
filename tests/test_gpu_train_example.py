"""The example run: 4-bit products, 8-bit moments, snapshots, and a restart that ends in the same bits; its loss falls."""
import re

import pytest

from paper_2406_10707_amd import train_example

pytestmark = pytest.mark.gpu


def test_the_run_learns_and_restarts_bit_for_bit(capsys):
    print("training example", flush=True)
    assert train_example.main(["--steps", "60", "--every", "20"]) == 0
    out = capsys.readouterr().out
    losses = [float(x) for x in re.findall(r"loss ([\d.]+)", out)]
    assert len(losses) == 4 and losses[-1] < 0.5 * losses[0], losses
    assert "6.06 bytes a parameter" in out and "the same, bit for bit" in out
