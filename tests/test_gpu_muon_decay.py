"""What a rate of a matrix's own does to its decay: it has it too, and weight_decay = d / lr_scale leaves a decay of lr * d."""
import math

import pytest
import torch

import matrix_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_matrices import F32, low_rank, randn, run_muon, update_of

pytestmark = pytest.mark.gpu

LR, DECAY = 0.05, 0.4


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


@pytest.mark.parametrize("steps", [0, 5])
@pytest.mark.parametrize("shapes", [[(160, 20), (20, 160), (40, 40)], [(800, 100), (100, 800), (400, 400), (66, 65)]])
def test_decay_of_matrices_with_a_rate_of_their_own(det, shapes, steps):
    """Tiny matrices, and larger ones; with 5 steps and with none."""
    mats = [(low_rank(*s, 3 * i), low_rank(*s, 3 * i + 1)) for i, s in enumerate(shapes)]
    start = [randn(s, i, F32, 0.5) for i, s in enumerate(shapes)]
    scales = [math.sqrt(max(1.0, r / c)) for r, c in shapes]
    for decays, of in ((DECAY, lambda s: LR * s * DECAY), ([DECAY / s for s in scales], lambda s: LR * DECAY)):
        params, _, _ = run_muon(det, mats, param=[p.cuda() for p in start], lr=LR, lr_scale=scales, weight_decay=decays, steps=steps)
        for (g, m), p0, p, s in zip(mats, start, params, scales):
            up = update_of(g, m)[1]
            exact, bound = refs.orthogonal_bound(up, "f32") if steps else (up.double() / (float(torch.linalg.matrix_norm(up.double())) + 1e-7), 2.0 ** -20)
            want = p0.double() * (1 - of(s)) - LR * s * exact
            # (the two factors, two products, a difference and the rounding in fp32, beside what X is off by)
            may = 5 * refs.U32 * (p0.double().abs() + LR * s * exact.abs()) + LR * s * bound
            assert bool(((p.double().cpu() - want).abs() <= may).all()), (tuple(p.shape), decays)
