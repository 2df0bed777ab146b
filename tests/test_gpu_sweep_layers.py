"""The sweep's training step with layers, as the example runs it: it repeats bit for bit, its gradients are those of its packed
numbers, and its rates are scored."""
import os
import sys

import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import sweep_step  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("products", ["f32", "f16"])
def test_step_repeats(products):
    det = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    step = sweep_step.LayerStep(det, 300, 1000, 136, 32, layers=3, products=products)
    rates, losses, first = sweep_step.measure(step, 5)
    assert all(r > 0 for r in rates.values()) and set(rates) == set(step.parts)
    _, again, second = sweep_step.measure(step, 5)
    assert losses == again and first == second
    step.masters[1].view(-1)[123] += 1e-3                              # one wrong number
    assert step.checksum() != first
    det.close()


def test_gradients_of_a_step():
    det = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    step = sweep_step.LayerStep(det, 300, 1000, 136, 32, layers=2)
    step.reset()
    step.lookup()
    step.forward()
    step.loss()
    value = lambda p: refs.values(p["codes"], p["exp"].cpu())                                   # noqa: E731
    x, w = value(step.packed_hidden[0][0]), value(step.packed_weight[0][0])
    ref, bound = refs.product(x, w, torch.bfloat16, step.input.cpu())
    assert bool(((step.hiddens[0].double().cpu() - ref).abs() <= bound).all())
    before = step.grad["hidden"].clone()
    step.backward()
    # the first layer's are the last that `packed_grad` held: of dy what it was packed from is gone, of its numbers all is there
    dyt, xt = value(step.packed_grad[1]), value(step.packed_hidden[0][1])
    ref, bound = refs.product(dyt, xt, torch.float32)
    assert bool(((step.weight_grads[0].double().cpu() - ref).abs() <= bound).all())
    dy, wt = value(step.packed_grad[0]), value(step.packed_weight[0][1])
    ref, bound = refs.product(dy, wt, torch.bfloat16)
    # (dy itself is added: packing has rounded it by half a step of e4m3 at most, 2^-4, or of its smallest numbers, 2^-10 of the block's unit)
    off = (step.grad["hidden"].double().cpu() - ref - dy).abs()
    unit = torch.exp2(step.packed_grad[0]["exp"].cpu().double() - 127).t().repeat_interleave(128, 1)[:, :136]
    # (what e4m3 holds lies within 1 + 2^-4 of the number)
    assert bool((off <= bound + dy.abs() * 2.0 ** -3 + unit * 2.0 ** -9 + 2.0 ** -8 * (ref + dy).abs() * 2).all())
    assert not torch.equal(before, step.grad["hidden"])
    det.close()


def test_example_runs(capsys):
    assert sweep_step.main(["--rows", "256", "--vocab", "2000", "--width", "128", "--layers", "2", "--steps", "3", "--tolerance", "1e9"]) == 0
    out = capsys.readouterr().out
    assert "same bits" in out and all(p in out for p in sweep_step.LayerStep.parts)
