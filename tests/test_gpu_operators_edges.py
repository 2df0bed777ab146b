"""More of the operators of a sweep's own training step against 64 bits, at the sizes, types and values that the tests
beside this one leave out; bounds as derived in operator_refs.py."""
import pytest
import torch

import operator_refs as refs
from paper_2605_17879_amd import Config, Detector
from test_gpu_operators import BF16, F16, F32, check_grad, check_loss, poison, randn, run_loss, say, within

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


PROBABLE = [(9, 300, 64), (20, 70000, 72), (70, 1500, 72), (300, 5001, 64), (2100, 9001, 72)]


def probable_targets(n, vocab, d, dtype, near=False):
    """Hidden states, weights and targets that are probable: 24 words share most of each row's probability.  Column c of the
    first 24 is 1.5 for the c-th of those words and 0 for all others, so that an element of the hidden states'
    gradient there is one element of G times 1.5.  near: the 24 words are the first ones."""
    some = torch.arange(24) if near else torch.randperm(vocab, generator=torch.Generator().manual_seed(5))[:24]
    h, w = randn((n, d), 1, dtype), randn((vocab, d), 2, dtype, 0.1)
    w[some] = randn((24, d), 3, dtype, 2 / d ** 0.5)
    w[:, :24] = 0
    w[some, torch.arange(24)] = 1.5
    # (5 to 9 above the other words' logits, whose number that makes up for)
    h[:, -1] = 1.0
    w[:, -1] = 0
    w[some, -1] = 3.0 + float(torch.tensor(vocab).log2()) / 2
    which = torch.multinomial(torch.softmax(h.double() @ w[some].double().T, 1), 1, generator=torch.Generator().manual_seed(6))[:, 0]
    return h, w, some, which


def target_element(ref, h, w, t, c, dtype, left_out=0.0):
    """G at the rows' targets where what rounding drops there is kept, rounded to the type itself: its value, and how far off it
    may be (the exponent's error, the exponential's, the subtraction's and products', the square of a rounding, and what is
    left out for being little)."""
    n = len(t)
    logits = (h.double() @ w.double().T)[torch.arange(n), t]
    p = torch.exp(logits - ref.lse)
    expo = ref.logit_err[torch.arange(n), t] + ref.lse_bound + 4 * refs.U32 * (logits.abs() + ref.lse.abs())
    g = c * (p - 1)
    err = abs(c) * p * (torch.expm1(expo) + 4 * refs.U32) + (refs.u(dtype) ** 2 + left_out + 6 * refs.U32) * g.abs() * (1 + expo)
    return p, g, err + (abs(c) * 2.0 ** -38 if dtype == F16 else 0.0)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,vocab,d", PROBABLE)
def test_hidden_gradient_at_probable_targets_is_rounded_once(det, dtype, n, vocab, d):
    """One product, its addition to zeros, what the rounding of G drops, two factors: eight roundings to fp32, one to the type."""
    say(f"probable targets, hidden: {dtype} n={n} vocab={vocab} d={d}")
    h, w, some, which = probable_targets(n, vocab, d, dtype)
    t = some[which]
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    p, g, err = target_element(ref, h, w, t, 1.0 / n, dtype)
    assert float(((p > 0.05) & (p < 0.95)).double().mean()) > 0.3, "the targets are not what the test is about"
    out = run_loss(det, h, w, t, grad_mean=1.0)
    want = 1.5 * g
    err = 1.5 * err + 8 * refs.U32 * want.abs()
    low = torch.finfo(dtype).smallest_normal * refs.u(dtype) * 2
    within(out["hidden_grad"].cpu()[torch.arange(n), which], want, err + refs.u(dtype) * (want.abs() + err) + low, "gradient at the target")
    within(out["hidden_grad"], ref.hidden_grad, ref.hidden_grad_bound, "gradient of the hidden states")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,vocab,near", [(24, 300, False), (40, 300, False), (70, 1500, False), (200, 33001, False), (300, 5001, False), (2100, 9001, False),
                                          (2100, 9001, True), (2100, 9100, True), (200, 200, True)])
def test_weights_gradient_at_probable_targets_is_rounded_once(det, dtype, n, vocab, near):
    """Columns in which one row's hidden state is 1.5 and all others are 0: the target's gradient there is one element of G times
    1.5.  Up to 2 100 rows have their targets in one tile, in several or in none.  What rounding drops counts from a sixteenth of
    the most that it may drop on."""
    d = 264
    say(f"probable targets, weights: {dtype} n={n} vocab={vocab} near={near}")
    h, w, some, which = probable_targets(n, vocab, d, dtype, near)
    rows = torch.arange(n)[::max(1, n // 200)][:200]
    at = 24 + torch.arange(len(rows))
    h[:, 24:224] = 0
    h[rows, at] = 1.5
    t = some[which]
    t[3] = -1
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    keep = t[rows] >= 0
    rows, at = rows[keep], at[keep]
    part = refs.Loss(h[rows], w, t[rows])
    p, g, err = target_element(part, h[rows], w, t[rows], 1.0 / ref.count, dtype, refs.u(dtype) / 16)
    out = run_loss(det, h, w, t, grad_mean=1.0)
    want = 1.5 * g
    err = 1.5 * err + 8 * refs.U32 * want.abs()
    low = torch.finfo(dtype).smallest_normal * refs.u(dtype) * 2
    within(out["weight_grad"].cpu()[t[rows], at], want, err + refs.u(dtype) * (want.abs() + err) + low, "gradient at the target")
    within(out["weight_grad"], ref.weight_grad, ref.weight_grad_bound, "gradient of the weights")


@pytest.mark.parametrize("n,width", [(1 << 22, 4), (3_000_001, 3), (131_073, 8), (131_072, 8)])
def test_lookup_grad_of_a_token_over_millions_of_rows(det, n, width):
    """All rows are one token's, and their values alike, so that every addition's error goes the same way: the sum is as far off
    as its longest chain of additions allows, a stretch of at most 32 rows or a 4 096th of them, and a sixteenth of
    4 096 parts' with four levels of pairs in front of them."""
    say(f"one token, n={n}")
    vocab, value = 9, 1.9
    t = torch.full((n,), 3, device="cuda")
    g = torch.full((n, width), value, device="cuda")
    w = poison(torch.empty((vocab, width), device="cuda"))
    det.embed_grad(g, t, w, det.alloc_embed_grad_work(n, vocab, width), scale=0.5)
    chain = max(32, -(-n // (4096 * 8)) * 8) + 256 + 4 + 2
    want = torch.full((width,), float(torch.tensor(value)) * n * 0.5, dtype=torch.float64)
    within(w[3], want, chain * refs.U32 * want, "gradient")
    assert bool((w[torch.arange(vocab) != 3] == 0).all())


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,vocab,width", [(200_003, 2, 24), (150_000, 70_000, 8), (400_001, 40, 9)])
def test_lookup_grad_of_long_lists(det, accumulate, n, vocab, width):
    say(f"lookup_grad n={n} vocab={vocab} width={width} accumulate={accumulate}")
    t = refs.tokens(n, vocab, n + 1, padding=0.1)
    check_grad(det, randn((n, width), n, F32), t, vocab, 1.7, accumulate, randn((vocab, width), n + 2, F32))


@pytest.mark.parametrize("n,vocab,width,gap,padding", [
    (2100, 9001, 72, 0, 0.1), (22000, 130, 520, 0, 0.3), (40, 33001, 264, 0, 0.0), (2305, 8000, 200, 8, 0.0), (2049, 8191, 33, 0, 0.5),
])
def test_loss_and_gradients_in_large_tiles_of_f16(det, n, vocab, width, gap, padding):
    say(f"large tiles f16 n={n} vocab={vocab} width={width} gap={gap} padding={padding}")
    h, w = randn((n, width), n + width, F16), randn((vocab, width), n + vocab, F16, 2 / width ** 0.5)
    t = refs.tokens(n, vocab, n, padding)
    check_loss(run_loss(det, h, w, t, gap, grad_mean=1.0), refs.Loss(h, w, t, grad_mean=1.0))


@pytest.mark.parametrize("n,vocab,width,padding", [(1, 66001, 40, 0.0), (17, 70003, 136, 0.3), (33, 66001, 64, 0.1), (65, 66001, 72, 0.0), (9, 95, 2056, 0.0),
                                                   (64, 1090, 1000, 0.2)])
def test_loss_and_gradients_of_few_rows_of_f16(det, n, vocab, width, padding):
    say(f"few rows f16 n={n} vocab={vocab} width={width} padding={padding}")
    h, w = randn((n, width), n + width, F16), randn((vocab, width), n + vocab, F16, 2 / width ** 0.5)
    t = refs.tokens(n, vocab, n, padding)
    check_loss(run_loss(det, h, w, t, grad_mean=1.0), refs.Loss(h, w, t, grad_mean=1.0))


@pytest.mark.parametrize("scale", [-0.75, 0.0])
@pytest.mark.parametrize("n,vocab,width", [(9, 300, 64), (300, 5001, 72), (2100, 9001, 72)])
def test_logit_scales_below_one_of_f16(det, scale, n, vocab, width):
    h, w, t = randn((n, width), 1, F16), randn((vocab, width), 2, F16, 0.5), refs.tokens(n, vocab, 3, 0.1)
    check_loss(run_loss(det, h, w, t, 0, scale, grad_mean=1.0), refs.Loss(h, w, t, scale, grad_mean=1.0))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("grad_mean", [1.0, 2.0 ** 10])
@pytest.mark.parametrize("n,vocab,width", [(2500, 3000, 40), (2100, 9001, 72)])
def test_small_probabilities_have_their_part_in_the_gradients(det, dtype, grad_mean, n, vocab, width):
    """A mean over thousands of rows: where G is not taken relative to the largest coefficient, the words without a target
    have one of a few of f16's least numbers, and the bound on its rounding is passed."""
    h, w = randn((n, width), 1, dtype), randn((vocab, width), 2, dtype, 0.1)
    t = refs.tokens(n, vocab // 2, 3)                               # (the second half is no row's target)
    ref = refs.Loss(h, w, t, grad_mean=grad_mean)
    out = run_loss(det, h, w, t, grad_mean=grad_mean)
    check_loss(out, ref)
    others = out["weight_grad"][vocab // 2:].double().cpu()
    assert float((others != 0).double().mean()) > 0.95


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_table_keeps_the_memory_that_it_updates(det, bits):
    """Storages exchanged behind a table: the update by it goes to the old memory, which nobody else has got meanwhile."""
    n = 3_000_001
    make = lambda: torch.ones(n, device="cuda")                      # noqa: E731
    p, g, c = make(), make(), torch.zeros(n, dtype=BF16, device="cuda")
    state = det.alloc_adamw_state([p], bits)
    table = det.adamw_table([p], [g], state, copies=[c])
    tensors = [p, g, c] + [x[0] for x in state.values()]
    old = {t.data_ptr() for t in tensors}
    for t in tensors:
        t.data = torch.zeros(8, dtype=t.dtype, device="cuda")
    others = [torch.full((n,), 7, dtype=t.dtype, device="cuda") for t in tensors[:5] for _ in range(2)]
    assert not old & {t.data_ptr() for t in others}
    det.adamw(table, lr=1e-2, step=1)
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in others)


def test_adamw_with_another_table_size_writes_nothing(det):
    p, g = [torch.ones(1000, device="cuda") for _ in range(40)], [torch.ones(1000, device="cuda") for _ in range(40)]
    state = det.alloc_adamw_state(p)
    table = det.adamw_table(p, g, state)
    assert table["bytes"].numel() > 512
    det.adamw({"bytes": table["bytes"][:512]}, lr=1e-2, step=1)
    assert all(bool((t == 1).all()) for t in p) and all(bool((t == 0).all()) for v in state.values() for t in v)
    det.adamw(table, lr=1e-2, step=1)
    assert all(bool((t < 1).all()) for t in p)


@pytest.mark.parametrize("n,vocab,d,gap,dtype", [
    # rows apart and unaligned, copied in one piece and in two; G in two pieces
    (70, 1500, 264, 3, F16), (300, 5001, 264, 8, BF16), (70, 70_000, 2056, 3, BF16), (9, 70_000, 2056, 3, BF16), (20, 300, 264, 3, F16),
    (4200, 66_001, 264, 0, BF16), (4200, 66_001, 264, 0, F16), (2100, 9001, 265, 0, BF16),
])
def test_gradients_at_probable_targets_over_pieces(det, n, vocab, d, gap, dtype):
    """The elements of the two tests before, with coefficients of each row's own, a logit scale, rows left out, and operands that lie and
    are cut in other ways."""
    say(f"probable targets over pieces: {dtype} n={n} vocab={vocab} d={d} gap={gap}")
    h, w, some, which = probable_targets(n, vocab, d, dtype)
    w = w * 2                                                        # (exact, and undone by the scale)
    picked = torch.arange(n)[::max(1, n // 60)][:60]
    at = 24 + torch.arange(len(picked))
    h[:, 24:224] = 0
    h[picked, at] = 1.5
    t = some[which]
    t[3::7] = -1
    coef = randn((n,), 8, F32, 0.5) + 1.0
    out = run_loss(det, h, w, t, gap, 0.5, grad_mean=0.75, grad_rows=coef)
    keep = t[picked] >= 0
    picked, at, which = picked[keep], at[keep], which[picked[keep]]
    ref = refs.Loss(h[picked], w, t[picked], 0.5)
    c = coef[picked].double() + 0.75 / int((t >= 0).sum())
    most = float(coef.abs().max()) + 1.0
    logits = 0.5 * (h[picked].double() @ w.double().T)[torch.arange(len(picked)), t[picked]]
    p = torch.exp(logits - ref.lse)
    expo = ref.logit_err[torch.arange(len(picked)), t[picked]] + ref.lse_bound + 4 * refs.U32 * (logits.abs() + ref.lse.abs())
    g = c * (p - 1)
    low = torch.finfo(dtype).smallest_normal * refs.u(dtype) * 2
    for name, i, j, factor, left_out in (("hidden_grad", picked, which, 1.5, 0.0), ("weight_grad", t[picked], at, 0.75, refs.u(dtype) / 16)):
        want = factor * g
        err = c.abs() * p * (torch.expm1(expo) + 4 * refs.U32) + (refs.u(dtype) ** 2 + left_out + 6 * refs.U32) * g.abs() * (1 + expo)
        err = factor * (err + (most * 2.0 ** -38 if dtype == F16 else 0.0)) + 8 * refs.U32 * want.abs()
        within(out[name].cpu()[i, j], want, err + refs.u(dtype) * (want.abs() + err) + low, name)
    assert bool((out["hidden_grad"][(t < 0).cuda()] == 0).all())
