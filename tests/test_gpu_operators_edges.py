"""More of the operators of a sweep's own training step against 64 bits, at the sizes, types and values that the tests
beside this one leave out; bounds as derived in operator_refs.py."""
import pytest
import torch

import operator_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_operators import BF16, randn, run_loss, say, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


@pytest.mark.parametrize("n,gap", [(68942, 0), (69326, 3)])
def test_loss_of_more_tiles_than_a_launch_holds(det, n, gap):
    """More than 2^37 logits: the vocabulary is cut into launches, and every word counts once, those at a cut too.  The last
    word of each 128 in the last 20 000 and the first word behind it stand out, so that one counted twice, or 129
    times, shows in each row."""
    V, d = 2_000_000, 8
    say(f"loss over {V} words for {n} rows")
    h, w = randn((n, d), 1, BF16), randn((V, d), 2, BF16, 0.05)
    h[:, 0] = 4.0
    raised = torch.arange(V - 20_000, V)
    w[raised[(raised % 128 == 127) | (raised % 128 == 0)], 0] = 3.0
    t = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(3))
    t[::2] = raised[torch.arange(len(t[::2])) % len(raised)]
    out = run_loss(det, h, w, t, gap, grad=False)
    rows = torch.arange(0, n, n // 40)
    ref = refs.Loss(h[rows], w, t[rows])
    within(out["lse"][rows.cuda()], ref.lse, ref.lse_bound, "lse")
    within(out["loss"][rows.cuda()], ref.loss, ref.loss_bound, "loss")
    assert float(out["mean"][1]) == n
    assert abs(float(out["mean"][0]) - float(out["loss"].double().mean())) < 1e-5 * float(out["mean"][0])


@pytest.mark.parametrize("n,vocab,width", [(9, 300, 64), (300, 5001, 72), (2100, 9001, 72)])
def test_a_logit_scale_that_is_no_number(det, n, vocab, width):
    """Every logit is none then, and so is all that comes of them: sums, losses, the gradients' rows that have one."""
    h, w, t = randn((n, width), 1, BF16), randn((vocab, width), 2, BF16, 0.5), refs.tokens(n, vocab, 3, 0.2)
    out = run_loss(det, h, w, t, 0, float("nan"), grad_mean=1.0)
    keep = (t >= 0).cuda()
    assert bool(torch.isnan(out["lse"]).all())
    assert bool(torch.isnan(out["loss"][keep]).all()) and bool((out["loss"][~keep] == 0).all()) and bool(torch.isnan(out["mean"][0]))
    assert bool(torch.isnan(out["hidden_grad"][keep]).all()) and bool((out["hidden_grad"][~keep] == 0).all())
    assert bool(torch.isnan(out["weight_grad"]).all())
