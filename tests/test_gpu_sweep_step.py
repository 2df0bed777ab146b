"""The sweep's own training step as the example runs it: it learns, repeats bit for bit, and its rates are scored."""
import os
import sys

import pytest
import torch

from paper_2605_17879_amd import Config, Detector

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import sweep_step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_step_learns_and_repeats(bits):
    det = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    step = sweep_step.SweepStep(det, 500, 3000, 264, bits)
    rates, losses, first = sweep_step.measure(step, 30)
    assert losses[-1] < losses[0] - 0.5 and all(r > 0 for r in rates.values())
    _, again, second = sweep_step.measure(step, 30)
    assert losses == again and first == second
    step.master.view(-1)[12345] += 1e-3                                # one wrong number
    assert step.checksum() != first
    det.close()


def test_example_runs(capsys):
    assert sweep_step.main(["--rows", "256", "--vocab", "2000", "--width", "128", "--steps", "3", "--tolerance", "1e9"]) == 0
    out = capsys.readouterr().out
    assert "same bits" in out and all(p in out for p in sweep_step.PARTS)
