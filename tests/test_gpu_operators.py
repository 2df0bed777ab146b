"""The operators of a sweep's own training step (lookup, cross entropy over a projected vocabulary, their
gradients, AdamW) against plain implementations in 64 bits, at the sizes and masks where they can go
wrong; every bound is derived in operator_refs.py from the roundings that the kernels make."""
import numpy as np
import pytest
import torch

import operator_refs as refs
from paper_2605_17879_amd import Config, Detector

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def det():
    d = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1))
    yield d
    d.close()


def say(text):
    print(text, flush=True)


def randn(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def spaced(t, gap, at=0):
    """t on the GPU with `gap` elements between the end of a row and the next, `at` elements into its storage."""
    if gap == 0 and at == 0:
        return t.cuda()
    n, d = t.shape
    store = torch.full((n * (d + gap) + at + 16,), float("nan"), dtype=t.dtype, device="cuda")
    view = store[at:at + n * (d + gap)].view(n, d + gap)[:, :d]
    view.copy_(t)
    return view


def poison(t):
    t.view(torch.uint8).fill_(0xA5) if t.is_contiguous() else t.fill_(float("nan"))
    return t


def within(got, ref, bound, what):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    off = (got - ref).abs().nan_to_num()
    worst = (off - bound.nan_to_num()).max() if off.numel() else torch.tensor(0.0)
    assert off.numel() == 0 or bool((off <= bound.nan_to_num(posinf=0)).all()), f"{what}: off by {float(worst):.3g} more than may be"


# ---- lookup ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,vocab,width,gap,at", [
    (1, 1, 1, 0, 0), (1, 7, 4096, 0, 0), (3, 100, 8, 0, 0), (65, 1000, 33, 0, 0), (257, 50, 24, 8, 0), (130, 333, 1000, 0, 0),
    (64, 99, 256, 3, 0), (31, 99, 64, 0, 1), (1000, 40, 2056, 0, 0),
])
def test_lookup(det, dtype, n, vocab, width, gap, at):
    say(f"lookup {dtype} n={n} vocab={vocab} width={width} gap={gap} at={at}")
    w = randn((vocab, width), n + width, dtype)
    for kind in (torch.int64, torch.int32):
        t = refs.tokens(n, vocab, n, padding=0.2, dtype=kind)
        if n > 2:
            t[n // 2] = vocab + 5                                  # no row of the table
        out = poison(torch.empty((n, width), dtype=dtype, device="cuda"))
        det.embed(spaced(w, gap, at), t.cuda(), out, scale=2.5)
        want = refs.lookup(w, t, 2.5)
        assert torch.equal(out.cpu().nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))


def test_lookup_of_nothing(det):
    w = randn((5, 16), 1, F32).cuda()
    det.embed(w, torch.zeros(0, dtype=torch.int64, device="cuda"), torch.empty((0, 16), device="cuda"))
    out = torch.empty((3, 16), device="cuda")
    det.embed(torch.empty((0, 16), device="cuda"), torch.tensor([-1, 0, 3], device="cuda"), out)
    assert torch.equal(out[0].cpu(), torch.zeros(16)) and bool(torch.isnan(out[1:]).all())


def test_lookup_with_strided_tokens_and_output(det):
    w = randn((50, 40), 2, BF16)
    t = refs.tokens(2 * 33, 50, 3)
    out = torch.full((33, 64), 9.0, dtype=BF16, device="cuda")
    det.embed(w.cuda(), t.cuda()[::2], out[:, :40])
    assert torch.equal(out[:, :40].cpu(), refs.lookup(w, t[::2], 1.0)) and bool((out[:, 40:] == 9).all())


# ---- its gradient ----------------------------------------------------------------------------------

def check_grad(det, g, t, vocab, scale, accumulate, old=None, gap=0):
    n, width = g.shape
    w = spaced(old, gap) if accumulate else poison(torch.empty((vocab, width), dtype=g.dtype, device="cuda"))
    work = poison(det.alloc_embed_grad_work(n, vocab, width))
    det.embed_grad(spaced(g, gap), t.cuda(), w, work, scale=scale, accumulate=accumulate)
    ref, bound = refs.lookup_grad(g, t, scale, vocab, old if accumulate else None)
    untouched = torch.bincount(t[(t >= 0) & (t < vocab)].long(), minlength=vocab) == 0
    first = w.clone()
    assert torch.equal(first[untouched.cuda()].cpu(), old[untouched] if accumulate else torch.zeros_like(ref[untouched]).to(g.dtype))
    within(first, ref, bound, "gradient")
    if accumulate:
        w.copy_(old)
    det.embed_grad(spaced(g, gap), t.cuda(), w, work, scale=scale, accumulate=accumulate)
    assert torch.equal(first, w), "a second pass differs"


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,vocab,width,gap", [
    (1, 1, 1, 0), (1, 300, 64, 0), (31, 2, 40, 0), (32, 70000, 8, 0), (33, 5, 1000, 0), (97, 1000, 33, 0), (500, 257, 256, 8),
    (4097, 600, 130, 0), (9000, 90, 24, 0), (20000, 300, 32, 0), (70001, 2000, 8, 0),
])
def test_lookup_grad(det, accumulate, dtype, n, vocab, width, gap):
    say(f"lookup_grad {dtype} n={n} vocab={vocab} width={width} gap={gap} accumulate={accumulate}")
    t = refs.tokens(n, vocab, n + 1, padding=0.1, dtype=torch.int32 if n % 2 else torch.int64)
    if n > 40:
        t[7], t[20] = vocab, vocab + 1000                          # no rows: no part in it
    check_grad(det, randn((n, width), n, dtype), t, vocab, 1.7, accumulate, randn((vocab, width), n + 2, dtype), gap)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,vocab,width,dtype", [
    # both sides of the lines between lists that are compared, sorted at once, by workgroups that count all, and by ones that do not
    (1024, 3000, 520, BF16), (1024, 40, 33, F32), (1025, 3000, 136, BF16), (2048, 50, 72, F16), (2049, 3000, 24, F32), (3000, 70000, 24, F16), (4096, 500, 72, F32),
    (65536, 600, 8, BF16), (65537, 600, 8, BF16), (30000, 1 << 19, 8, F32),
    # few rows: wide ones, rows that are not aligned, more rows of the table than one workgroup marks
    (700, 90, 4096, F32), (1000, 50, 2500, F16), (900, 12, 1001, BF16), (9, 16385, 1, BF16), (300, 300000, 2, F32), (2, 1 << 20, 4, F32),
])
def test_lookup_grad_of_lists_of_all_lengths(det, accumulate, n, vocab, width, dtype):
    say(f"lookup_grad of lists {dtype} n={n} vocab={vocab} width={width} accumulate={accumulate}")
    t = refs.tokens(n, vocab, n + 1, padding=0.05)
    check_grad(det, randn((n, width), n, dtype), t, vocab, 0.7, accumulate, randn((vocab, width), n + 2, dtype))


@pytest.mark.parametrize("n", [9, 63, 64, 65, 700, 1024, 1500, 2048])
def test_lookup_grad_of_few_tokens_over_and_over(det, n):
    """One to three tokens in a list of few rows, in runs and in turn."""
    say(f"few tokens over and over, n={n}")
    i = torch.arange(n)
    for t in (torch.full((n,), 3), i % 2 * 4, torch.where(i < n // 2, 1, 2), torch.where(i % 3 == 0, -1, 5)):
        check_grad(det, randn((n, 264), n, BF16), t, 9, 1.0, False)
        check_grad(det, randn((n, 264), n, F32), t, 9, 1.5, True, randn((9, 264), 1, F32))


@pytest.mark.parametrize("n", [5, 5000])
@pytest.mark.parametrize("gap", [8, 3])
def test_lookup_grad_into_rows_apart(det, n, gap):
    """Zeros and sums stay inside the rows."""
    vocab, width = 333, 48
    t, g = refs.tokens(n, vocab, 4, 0.1), randn((n, width), 5, BF16)
    store = torch.full((vocab, width + gap), 9.0, dtype=BF16, device="cuda")
    det.embed_grad(g.cuda(), t.cuda(), store[:, :width], det.alloc_embed_grad_work(n, vocab, width), scale=0.5)
    ref, bound = refs.lookup_grad(g, t, 0.5, vocab)
    within(store[:, :width], ref, bound, "gradient")
    assert bool((store[:, width:] == 9).all())


@pytest.mark.parametrize("n", [32, 64, 95, 1000, 40000])
def test_lookup_grad_of_one_token(det, n):
    """Every row is the same token's: one sum over all stretches."""
    say(f"one token, n={n}")
    t = torch.full((n,), 3)
    check_grad(det, randn((n, 72), n, F32), t, 9, 1.0, False)
    check_grad(det, randn((n, 72), n, BF16), torch.where(torch.arange(n) < 32, torch.full_like(t, 2), t), 9, 1.0, False)


def test_lookup_grad_ignores_what_padded_rows_hold(det):
    t = refs.tokens(300, 20, 5, padding=0.5)
    g = randn((300, 48), 6, F32)
    clean = g.clone()
    g[t < 0] = float("nan")
    w = torch.empty((20, 48), device="cuda")
    det.embed_grad(g.cuda(), t.cuda(), w, det.alloc_embed_grad_work(300, 20, 48))
    ref, bound = refs.lookup_grad(clean, t, 1.0, 20)
    within(w, ref, bound, "gradient")


def test_lookup_grad_without_a_token(det):
    for t in (torch.zeros(0, dtype=torch.int64), torch.full((50,), -1)):
        w = torch.full((9, 16), 4.0, device="cuda")
        g = torch.zeros((len(t), 16), device="cuda")
        work = det.alloc_embed_grad_work(len(t), 9, 16)
        det.embed_grad(g, t.cuda(), w, work, accumulate=True)
        assert bool((w == 4).all())
        det.embed_grad(g, t.cuda(), w, work)
        assert bool((w == 0).all())


# ---- loss --------------------------------------------------------------------------------------

LOSSES = [
    # rows, vocabulary, width, gap, padding
    (1, 1, 1, 0, 0.0), (1, 2, 8, 0, 0.0), (1, 1000, 64, 0, 0.0), (2, 129, 72, 0, 0.0), (3, 1031, 200, 0, 0.3), (5, 4099, 1000, 0, 0.0),
    (17, 257, 33, 0, 0.2), (64, 128, 128, 0, 0.0), (100, 513, 136, 8, 0.5), (129, 300, 72, 3, 0.1), (130, 127, 8, 0, 0.0),
    (257, 1500, 264, 0, 0.3), (300, 5001, 96, 0, 0.02), (513, 770, 520, 16, 0.0),
]


def run_loss(det, hidden, weight, t, gap=0, scale=1.0, grad=True, grad_mean=None, grad_rows=None, work=None):
    n, d = hidden.shape
    V = weight.shape[0]
    h, w, td = spaced(hidden, gap), spaced(weight, gap), t.cuda()
    out = {k: poison(v) for k, v in det.alloc_vocab_loss(n).items()}
    if work is None:
        work = poison(det.alloc_vocab_loss_work(n, V, d, grad=grad))
    det.vocab_loss(h, w, td, out, work, logit_scale=scale)
    if not grad:
        return out
    g = {"hidden": poison(torch.empty((n, d), dtype=hidden.dtype, device="cuda")),
         "weight": poison(torch.empty((V, d), dtype=hidden.dtype, device="cuda"))}
    det.vocab_loss_grad(h, w, td, out, g, work, grad_mean=None if grad_mean is None else torch.tensor([grad_mean], device="cuda"),
                        grad_rows=None if grad_rows is None else grad_rows.cuda(), logit_scale=scale)
    return {**out, "hidden_grad": g["hidden"], "weight_grad": g["weight"]}


def check_loss(out, ref, grad=True):
    within(out["lse"], ref.lse, ref.lse_bound, "lse")
    within(out["loss"], ref.loss, ref.loss_bound, "loss")
    within(out["mean"][:1], ref.mean.view(1), ref.mean_bound.view(1), "mean")
    assert float(out["mean"][1]) == ref.count
    if grad:
        within(out["hidden_grad"], ref.hidden_grad, ref.hidden_grad_bound, "gradient of the hidden states")
        within(out["weight_grad"], ref.weight_grad, ref.weight_grad_bound, "gradient of the weights")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,vocab,width,gap,padding", LOSSES)
def test_loss_and_gradients(det, dtype, n, vocab, width, gap, padding):
    say(f"loss {dtype} n={n} vocab={vocab} width={width} gap={gap} padding={padding}")
    h, w = randn((n, width), n + width, dtype), randn((vocab, width), n + vocab, dtype, 2 / width ** 0.5)
    t = refs.tokens(n, vocab, n, padding, torch.int32 if n % 2 else torch.int64)
    rows = randn((n,), n + 9, F32)
    ref = refs.Loss(h, w, t, 1.25, grad_mean=0.75, grad_rows=rows)
    out = run_loss(det, h, w, t, gap, 1.25, grad_mean=0.75, grad_rows=rows)
    check_loss(out, ref)
    again = run_loss(det, h, w, t, gap, 1.25, grad_mean=0.75, grad_rows=rows)
    assert all(torch.equal(out[k], again[k]) for k in out), "a second pass differs"


@pytest.mark.parametrize("n,vocab,width,gap,padding", [
    # enough tiles of 256 x 256 for every CU: of the logits, of the hidden states' gradient, of the weights'
    (2100, 9001, 72, 0, 0.1), (22000, 130, 520, 0, 0.3), (40, 33001, 264, 0, 0.0), (2305, 8000, 200, 8, 0.0), (2049, 8191, 33, 0, 0.5),
])
def test_loss_and_gradients_in_large_tiles(det, n, vocab, width, gap, padding):
    say(f"large tiles n={n} vocab={vocab} width={width} gap={gap} padding={padding}")
    h, w = randn((n, width), n + width, BF16), randn((vocab, width), n + vocab, BF16, 2 / width ** 0.5)
    t = refs.tokens(n, vocab, n, padding)
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    check_loss(run_loss(det, h, w, t, gap, grad_mean=1.0), ref)


@pytest.mark.parametrize("n,vocab,width,padding", [
    (1, 66001, 40, 0.0), (16, 65600, 72, 0.0), (17, 70003, 136, 0.3), (33, 66001, 64, 0.1), (64, 65537, 200, 0.0), (65, 66001, 72, 0.0),
    (16, 1057, 200, 0.0), (17, 1025, 584, 0.0), (64, 1090, 1000, 0.2), (9, 95, 2056, 0.0), (40, 65536, 72, 0.9),
])
def test_loss_and_gradients_of_few_rows(det, n, vocab, width, padding):
    """Up to 64 rows, with vocabularies on both sides of the line between 32 and 128 words a workgroup."""
    say(f"few rows n={n} vocab={vocab} width={width} padding={padding}")
    h, w = randn((n, width), n + width, BF16), randn((vocab, width), n + vocab, BF16, 2 / width ** 0.5)
    t = refs.tokens(n, vocab, n, padding)
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    check_loss(run_loss(det, h, w, t, grad_mean=1.0), ref)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_mean_over_many_rows_does_not_underflow(det, dtype):
    """c = 1 / rows and small probabilities: G is far below the least f16 number if it is not scaled."""
    n, V, d = 2500, 3000, 40
    h, w = randn((n, d), 1, dtype), randn((V, d), 2, dtype, 0.5)
    t = refs.tokens(n, V, 3)
    ref = refs.Loss(h, w, t, grad_mean=1e-4)
    out = run_loss(det, h, w, t, grad_mean=1e-4)
    check_loss(out, ref)
    assert float((out["weight_grad"] != 0).float().mean()) > 0.5 or dtype == F16


def test_rows_left_out_may_hold_anything(det):
    n, V, d = 200, 500, 64
    h, w, t = randn((n, d), 1, BF16), randn((V, d), 2, BF16, 0.3), refs.tokens(n, V, 3, padding=0.4)
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    dirty = h.clone()
    dirty[t < 0] = float("nan")
    dirty[(t < 0) & (torch.arange(n) % 2 == 0)] = float("inf")
    out = run_loss(det, dirty, w, t, grad_mean=1.0)
    keep = t >= 0
    within(out["loss"], ref.loss, ref.loss_bound, "loss")
    within(out["lse"][keep.cuda()], ref.lse[keep], ref.lse_bound[keep], "lse")
    within(out["hidden_grad"], ref.hidden_grad, ref.hidden_grad_bound, "hidden")
    within(out["weight_grad"], ref.weight_grad, ref.weight_grad_bound, "weight")


def test_no_row_counts_and_no_rows(det):
    V, d = 300, 64
    w = randn((V, d), 2, BF16)
    for n in (0, 1, 150):
        out = run_loss(det, randn((n, d), 1, BF16), w, torch.full((n,), -100), grad_mean=1.0)
        assert out["mean"].tolist() == [0.0, 0.0] and bool((out["loss"] == 0).all())
        assert bool((out["hidden_grad"] == 0).all()) and bool((out["weight_grad"] == 0).all())


def test_targets_outside_the_vocabulary(det):
    n, V, d = 40, 130, 32
    h, w, t = randn((n, d), 1, F16), randn((V, d), 2, F16, 0.3), refs.tokens(n, V, 3, padding=0.2)
    t[5], t[11] = V, V + 2 ** 31
    ref = refs.Loss(h, w, t, grad_rows=torch.ones(n))
    out = run_loss(det, h, w, t, grad_rows=torch.ones(n))
    check_loss(out, ref)
    assert bool(torch.isnan(out["loss"][5])) and bool(torch.isnan(out["mean"][0]))


def test_confident_rows_and_far_logits(det):
    """Logits of hundreds: the exponentials need the running maximum, and G is zero but for rounding."""
    n, V, d = 64, 700, 48
    h, w = randn((n, d), 1, BF16, 6.0), randn((V, d), 2, BF16, 6.0)
    t = (h.double() @ w.double().T).argmax(1)
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    check_loss(run_loss(det, h, w, t, grad_mean=1.0), ref)


@pytest.mark.parametrize("scale", [-0.75, 0.0])
@pytest.mark.parametrize("n,vocab,width", [(9, 300, 64), (300, 5001, 72), (2100, 9001, 72)])
def test_logit_scales_below_one(det, scale, n, vocab, width):
    """A negative scale turns the order of the logits round; a scale of 0 leaves them all alike."""
    h, w, t = randn((n, width), 1, BF16), randn((vocab, width), 2, BF16, 0.5), refs.tokens(n, vocab, 3, 0.1)
    ref = refs.Loss(h, w, t, scale, grad_mean=1.0)
    check_loss(run_loss(det, h, w, t, 0, scale, grad_mean=1.0), ref)


@pytest.mark.parametrize("n,vocab,gap", [(9, 300, (5, 0)), (300, 5001, (5, 0)), (2100, 9001, (5, 0)), (9, 300, (0, 5)), (300, 5001, (0, 5))])
def test_words_that_are_switched_off(det, n, vocab, gap):
    """A word whose logit is minus infinity, by the last element of its weights, counts for nothing; hidden states or
    weights alone are copied, and the copy's rows go on where the others end."""
    d = 72
    h, w, t = randn((n, d), 1, BF16), randn((vocab, d), 2, BF16, 0.3), refs.tokens(n, vocab - 1, 3)
    h[:, -1] = 1.0
    w[-1, -1] = float("-inf")
    ref = refs.Loss(h, w[:-1], t)
    out = det.alloc_vocab_loss(n)
    det.vocab_loss(spaced(h, gap[0]), spaced(w, gap[1]), t.cuda(), out, poison(det.alloc_vocab_loss_work(n, vocab, d)))
    check_loss(out, ref, grad=False)


@pytest.mark.parametrize("n,vocab", [(9, 300), (100, 3001), (300, 5001), (2100, 9001)])
def test_weights_gradient_with_words_that_are_switched_off(det, n, vocab):
    """A word whose logit is minus infinity has a gradient of zeros, whatever the number of rows (those that fill the last
    tile are not there); the other words' is the one without it."""
    d = 72
    h, w, t = randn((n, d), 1, BF16), randn((vocab, d), 2, BF16, 0.3), refs.tokens(n, vocab - 1, 3, padding=0.1)
    h[:, -1] = 1.0
    w[-1, -1] = float("-inf")
    ref = refs.Loss(h, w[:-1], t, grad_mean=1.0)
    out, work = det.alloc_vocab_loss(n), poison(det.alloc_vocab_loss_work(n, vocab, d, grad=True))
    g = {"weight": poison(torch.empty((vocab, d), dtype=BF16, device="cuda"))}
    det.vocab_loss(h.cuda(), w.cuda(), t.cuda(), out, work)
    det.vocab_loss_grad(h.cuda(), w.cuda(), t.cuda(), out, g, work, grad_mean=torch.ones(1, device="cuda"))
    within(g["weight"][:-1], ref.weight_grad, ref.weight_grad_bound, "gradient of the weights")
    assert bool((g["weight"][-1] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,vocab,width,padding", [(1, 300, 72, 0.0), (2, 3001, 136, 0.0), (16, 1057, 200, 0.2), (17, 1025, 64, 0.0), (32, 66001, 40, 0.1),
                                                   (9, 70003, 72, 0.0)])
def test_weights_gradient_of_few_rows_is_rounded_once(det, dtype, n, vocab, width, padding):
    """Up to 32 rows: G is held in two numbers, whose sum is off by the square of a rounding (and in f16 by half of the least
    number, in units of 2^-14 of the largest coefficient's power of two), so that the gradient's own rounding is all that counts."""
    h, w = randn((n, width), n + width, dtype), randn((vocab, width), n + vocab, dtype, 2 / width ** 0.5)
    t = refs.tokens(n, vocab, n, padding)
    ref = refs.Loss(h, w, t, grad_mean=1.0)
    out = run_loss(det, h, w, t, grad_mean=1.0)
    keep = t >= 0
    logits = h.double() @ w.double().T
    p = torch.exp(logits - ref.lse[:, None])
    c = keep.double()[:, None] / max(1, ref.count)
    expo = ref.logit_err + ref.lse_bound[:, None] + 4 * refs.U32 * (logits.abs() + ref.lse.abs()[:, None])
    g = p.clone()
    g[torch.arange(n)[keep], t[keep].long()] -= 1.0
    g_err = c * (p * (torch.expm1(expo) + 4 * refs.U32) + (refs.u(dtype) ** 2 + 6 * refs.U32) * g.abs() * (1 + expo))
    if dtype == F16:
        g_err = g_err + c.max() * 2.0 ** -25 * 2.0 ** -13
    e = g_err.T @ h.double().abs() + 66 * refs.U32 * ((c * g).abs() + g_err).T @ h.double().abs()
    low = torch.finfo(dtype).smallest_normal * refs.u(dtype) * 2
    within(out["weight_grad"], ref.weight_grad, e + refs.u(dtype) * (ref.weight_grad.abs() + e) + low, "gradient of the weights")


def test_strided_targets_and_gradients(det):
    n, V, d = 150, 700, 72
    h, w = randn((n, d), 1, BF16), randn((V, d), 2, BF16, 0.3)
    t = refs.tokens(2 * n, V, 3, 0.1)
    ref = refs.Loss(h, w, t[::2], grad_mean=1.0)
    out, work = det.alloc_vocab_loss(n), det.alloc_vocab_loss_work(n, V, d, grad=True)
    det.vocab_loss(h.cuda(), w.cuda(), t.cuda()[::2], out, work)
    for gap, at in ((0, 0), (8, 0), (3, 0), (8, 1)):
        store = [torch.full((r * (d + gap) + at,), 9.0, dtype=BF16, device="cuda") for r in (n, V)]
        g = dict(zip(("hidden", "weight"), (s[at:].view(r, d + gap)[:, :d] for s, r in zip(store, (n, V)))))
        det.vocab_loss_grad(h.cuda(), w.cuda(), t.cuda()[::2], out, g, work, grad_mean=torch.ones(1, device="cuda"))
        check_loss({**out, "hidden_grad": g["hidden"], "weight_grad": g["weight"]}, ref)
        assert all(bool((s[at:].view(r, d + gap)[:, d:] == 9).all()) and bool((s[:at] == 9).all()) for s, r in zip(store, (n, V)))


def test_one_gradient_alone(det):
    n, V, d = 100, 400, 72
    h, w, t = randn((n, d), 1, BF16).cuda(), randn((V, d), 2, BF16, 0.3).cuda(), refs.tokens(n, V, 3).cuda()
    out, work = det.alloc_vocab_loss(n), det.alloc_vocab_loss_work(n, V, d, grad=True)
    det.vocab_loss(h, w, t, out, work)
    one = torch.ones(1, device="cuda")
    e = lambda r: torch.empty((r, d), dtype=BF16, device="cuda")
    both, a, b = {"hidden": e(n), "weight": e(V)}, {"hidden": e(n)}, {"weight": e(V)}
    for g in (both, a, b):
        det.vocab_loss_grad(h, w, t, out, g, work, grad_mean=one)
    assert torch.equal(both["hidden"], a["hidden"]) and torch.equal(both["weight"], b["weight"])


def test_gradient_against_differences(det):
    """The sum of weighted losses, moved along a direction on both sides: central differences of the
    kernel's own losses against its gradients.  Steps are powers of two and every moved value is a
    bf16 number, so that the inputs are exact; the losses are off by their bound each."""
    n, V, d = 24, 200, 32
    h = randn((n, d), 1, F32).mul(16).round().div(16).to(BF16)
    w = randn((V, d), 2, F32, 0.5).mul(16).round().div(16).to(BF16)
    t, rows = refs.tokens(n, V, 3), randn((n,), 4, F32)
    out = run_loss(det, h, w, t, grad_rows=rows)
    step = 2.0 ** -4
    for name, x in (("hidden_grad", h), ("weight_grad", w)):
        g = torch.Generator().manual_seed(9)
        direction = torch.randint(-1, 2, x.shape, generator=g).to(BF16)
        sides, second = [], []
        for sign in (1, -1):
            moved = x + sign * step * direction
            a, b = (moved, w) if name == "hidden_grad" else (h, moved)
            ref = refs.Loss(a, b, t)
            sides.append((run_loss(det, a, b, t, grad=False)["loss"].double().cpu() * rows).sum())
            second.append((ref.loss * rows).sum())
            bound = (ref.loss_bound * rows.abs()).sum()
        slope = (sides[0] - sides[1]) / (2 * step)
        along = (out[name].double().cpu() * direction.double()).sum()
        ref = refs.Loss(h, w, t, grad_rows=rows)
        # differences of the exact losses are off the exact slope by the third derivative's part, worked out here
        curve = abs((second[0] - second[1]) / (2 * step) - (getattr(ref, name) * direction.double()).sum())
        allowed = bound / step + curve + (getattr(ref, name + "_bound") * direction.double().abs()).sum()
        assert abs(slope - along) <= allowed, (name, float(slope), float(along), float(allowed))


# ---- AdamW -----------------------------------------------------------------------------------

def make_tensors(sizes, param, grad, bits, seed, at=0):
    """Tensors of these sizes, `at` elements into their storages, with states that have moved already."""
    out = dict(p=[], g=[], m=[], v=[], m_exp=[], v_exp=[])
    for i, n in enumerate(sizes):
        put = lambda x, k: torch.cat([torch.zeros(at, dtype=x.dtype), x]).cuda()[at:] if k else x.cuda()
        spread = torch.exp(2 * randn((n,), seed + 50 + i, F32))
        out["p"].append(put(randn((n,), seed + i, param, 0.1), at))
        out["g"].append(put((randn((n,), seed + 100 + i, F32, 1e-2) * spread).to(grad), at))
        m, r = randn((n,), seed + 200 + i, F32, 1e-3) * spread, randn((n,), seed + 300 + i, F32, 1e-2).abs() * spread
        if bits == 32:
            out["m"].append(put(m, at))
            out["v"].append(put(r * r, at))
        else:
            for k, x, root in (("m", m, False), ("v", r, True)):
                c, e = refs.encode(x.numpy(), np.zeros(n, dtype=np.uint32), root)
                out[k].append(put(torch.from_numpy(c), at))
                out[k + "_exp"].append(torch.from_numpy(e).cuda())
    return out


def as32(t):
    return t.float().cpu().numpy()


SIZES = [[1], [3], [0, 5, 0], [255], [256], [257], [4096], [4097, 1, 2, 70001, 12288, 300, 4095]]


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,copy", [(F32, F32, None), (F32, BF16, BF16), (BF16, BF16, None), (F16, F16, None), (F32, F16, F16)])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_adamw(det, sizes, param, grad, copy, bits, at):
    say(f"adamw {sizes} param={param} grad={grad} copy={copy} bits={bits} at={at}")
    x = make_tensors(sizes, param, grad, bits, 11, at)
    copies = None if copy is None else [torch.empty(n + at, dtype=copy, device="cuda")[at:] for n in sizes]
    state = {k: x[k] for k in (("m", "v", "m_exp", "v_exp") if bits == 8 else ("m", "v"))}
    decay = [0.1 if i % 2 == 0 else 0.0 for i in range(len(sizes))]
    rate = [1.0 + 0.5 * i for i in range(len(sizes))]
    first = [2 ** 32 - 100 + 1000 * i for i in range(len(sizes))]
    want = []
    for i, n in enumerate(sizes):
        host = [as32(x["p"][i]), as32(x["g"][i])]
        kw = dict(decay=decay[i], lr_scale=rate[i], first_index=first[i], grad_scale=0.75)
        if bits == 8:
            want.append((host, refs.adamw(*host, x["m"][i].cpu().numpy(), x["v"][i].cpu().numpy(), 1e-2, 5,
                                          m_exp=x["m_exp"][i].cpu().numpy(), v_exp=x["v_exp"][i].cpu().numpy(), **kw)))
        else:
            want.append((host, refs.adamw(*host, as32(x["m"][i]), as32(x["v"][i]), 1e-2, 5, **kw)))
    table = det.adamw_table(x["p"], x["g"], state, copies=copies, weight_decay=decay, lr_scale=rate, first_index=first)
    det.adamw(table, lr=1e-2, step=5, grad_scale=torch.tensor([0.75], device="cuda"))
    for i, (_, ref) in enumerate(want):
        p = torch.from_numpy(ref[0])
        assert torch.equal(x["p"][i].cpu(), p.to(param)), f"tensor {i}: parameters"
        if copy is not None:
            assert torch.equal(copies[i].cpu(), p.to(copy)), f"tensor {i}: copy"
        for name, r in zip(("m", "v", "m_exp", "v_exp"), ref[1:]):
            assert np.array_equal(x[name][i].cpu().numpy(), r), f"tensor {i}: {name}"


def test_adamw_of_nothing(det):
    det.adamw(det.adamw_table([], [], {"m": [], "v": []}), lr=1e-2, step=1)
    e = torch.empty(0, device="cuda")
    det.adamw(det.adamw_table([e], [e], {"m": [e], "v": [e]}), lr=1e-2, step=1)
    torch.cuda.synchronize()


def test_adamw_against_64_bits(det):
    """Some fifteen roundings of relative size 2^-24 an element; m and the denominator are sums of
    terms whose magnitudes bound their errors."""
    x = make_tensors([50000], F32, F32, 32, 3)
    p, g, m, v = (as32(x[k][0]) for k in ("p", "g", "m", "v"))
    rp, rm, rv = refs.adamw64(p, g, m, v, 1e-2, 7, decay=0.1)
    det.adamw(det.adamw_table(x["p"], x["g"], {"m": x["m"], "v": x["v"]}, weight_decay=0.1), lr=1e-2, step=7)
    m_err = 4 * refs.U32 * (0.9 * np.abs(m.astype(np.float64)) + 0.1 * np.abs(g.astype(np.float64)))
    assert np.all(np.abs(as32(x["m"][0]) - rm) <= m_err)
    assert np.all(np.abs(as32(x["v"][0]) - rv) <= 6 * refs.U32 * rv)
    denom = np.sqrt(rv / (1 - 0.999 ** 7)) + 1e-8
    move_err = 1e-2 / (1 - 0.9 ** 7) * (m_err + 12 * refs.U32 * np.abs(rm)) / denom
    assert np.all(np.abs(as32(x["p"][0]) - rp) <= move_err + 3 * refs.U32 * np.abs(p))


@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan")])
def test_adamw_writes_nothing_behind_an_overflow(det, scale):
    x = make_tensors([300, 5000], F32, BF16, 8, 4)
    before = {k: [t.clone() for t in x[k]] for k in x}
    table = det.adamw_table(x["p"], x["g"], {k: x[k] for k in ("m", "v", "m_exp", "v_exp")})
    det.adamw(table, lr=1e-2, step=1, grad_scale=torch.tensor([scale], device="cuda"))
    assert all(torch.equal(a, b) for k in x for a, b in zip(x[k], before[k]))


def test_adamw_blocks_of_zeros_and_of_infinities(det):
    n = 256 * 6 + 9
    x = make_tensors([n], F32, F32, 8, 5)
    x["g"][0][:] = 0
    for k in ("m", "v", "m_exp", "v_exp"):
        x[k][0][:] = 0
    x["g"][0][256 + 3] = float("inf")
    x["g"][0][512 + 3] = float("nan")
    x["g"][0][768:1024] = 1e-30                                    # a root of 1e-30 * sqrt(0.001): far from underflow
    x["g"][0][1024:1280] = 1e18
    host = [as32(x["p"][0]), as32(x["g"][0])] + [x[k][0].cpu().numpy() for k in ("m", "v")]
    ref = refs.adamw(*host, 1e-2, 1, m_exp=x["m_exp"][0].cpu().numpy(), v_exp=x["v_exp"][0].cpu().numpy())
    table = det.adamw_table(x["p"], x["g"], {k: x[k] for k in ("m", "v", "m_exp", "v_exp")})
    det.adamw(table, lr=1e-2, step=1)
    for name, r in zip(("m", "v", "m_exp", "v_exp"), ref[1:]):
        assert np.array_equal(x[name][0].cpu().numpy(), r), name
    assert x["m_exp"][0][:3].tolist() == [0, 255, 255]
    got = x["p"][0].cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref[0])) and np.array_equal(got[~np.isnan(got)], ref[0][~np.isnan(got)])


def test_eight_bit_means_keep_moving(det):
    """A root that grows by 0.05 % a step, far below half a code's step, follows its gradient: with
    rounding to the nearest code it would stand still.  After 400 steps the mean of 64 blocks' second
    moments is within 5 % of the exact one (a code is dithered 400 times by at most 1/8 of itself, and 16 384
    elements are averaged: the mean's error is below 1 % but for the products of dithered factors)."""
    n = 64 * 256
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 0.1, device="cuda")
    g[::256] = 1.0                                                 # each block's largest, ten times the others
    state = det.alloc_adamw_state([p], bits=8)
    table = det.adamw_table([p], [g], state)
    for step in range(1, 401):
        det.adamw(table, lr=0.0, step=step)
    r = refs.decode(state["v"][0].cpu().numpy(), state["v_exp"][0].cpu().numpy()).astype(np.float64)
    m = refs.decode(state["m"][0].cpu().numpy(), state["m_exp"][0].cpu().numpy()).astype(np.float64)
    rest = np.arange(n) % 256 != 0
    want = 0.01 * (1 - 0.999 ** 400)
    assert abs(np.mean(r[rest] ** 2) / want - 1) < 0.05
    assert abs(np.mean(m[rest]) / 0.1 - 1) < 0.05


# ---- streams, graphs, far offsets ------------------------------------------------------------

def whole_step(det, s, stream=None):
    det.embed(s["weight"], s["tokens"], s["hidden"], stream=stream)
    det.vocab_loss(s["hidden"], s["weight"], s["targets"], s["out"], s["work"], stream=stream)
    det.vocab_loss_grad(s["hidden"], s["weight"], s["targets"], s["out"], s["grad"], s["work"], grad_mean=s["one"], stream=stream)
    det.embed_grad(s["grad"]["hidden"], s["tokens"], s["grad"]["weight"], s["lookup_work"], accumulate=True, stream=stream)
    det.adamw(s["table"], lr=1e-2, step=1, stream=stream)


def step_state(det, n=200, V=700, d=64):
    e = lambda r: torch.empty((r, d), dtype=BF16, device="cuda")
    s = dict(master=randn((V, d), 1, F32, 0.3).cuda(), tokens=refs.tokens(n, V, 2, 0.1).cuda(), targets=refs.tokens(n, V, 3, 0.1).cuda(),
             hidden=e(n), out=det.alloc_vocab_loss(n), work=det.alloc_vocab_loss_work(n, V, d, grad=True),
             grad={"hidden": e(n), "weight": e(V)}, one=torch.ones(1, device="cuda"), lookup_work=det.alloc_embed_grad_work(n, V, d))
    s["weight"] = s["master"].to(BF16)
    s["state"] = det.alloc_adamw_state([s["master"]], bits=8)
    s["table"] = det.adamw_table([s["master"]], [s["grad"]["weight"]], s["state"], copies=[s["weight"]], weight_decay=0.1)
    return s


def results(s):
    return [s["master"], s["weight"], s["hidden"], s["grad"]["hidden"], s["grad"]["weight"], *s["out"].values(), *s["state"]["m"],
            *s["state"]["v"], *s["state"]["m_exp"], *s["state"]["v_exp"]]


def test_a_stream_of_its_own(det):
    a, b = step_state(det), step_state(det)
    whole_step(det, a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    whole_step(det, b, stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(results(a), results(b)))


def test_captured_step(det):
    """The whole step in a graph, replayed four times with eager work in between, against eager steps."""
    a, b = step_state(det), step_state(det)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        whole_step(det, b)
    torch.cuda.synchronize()
    for i in range(4):
        whole_step(det, a)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(results(a), results(b))), f"replay {i}"
        assert float(a["out"]["mean"][0]) > 0


def test_offsets_beyond_32_bits(det):
    """Tables of more than 2^32 bytes and more than 2^31 elements: their last rows are looked up,
    updated and projected onto."""
    V, d = 600_000, 4096
    w = torch.zeros((V, d), dtype=BF16, device="cuda")
    last = randn((64, d), 1, BF16, 1 / 64).cuda()
    w[-64:] = last
    t = torch.arange(V - 64, V, device="cuda")
    out = torch.empty((64, d), dtype=BF16, device="cuda")
    det.embed(w, t, out)
    assert torch.equal(out, last)
    det.embed_grad(out, t, w, det.alloc_embed_grad_work(64, V, d), accumulate=True)
    assert torch.equal(w[-64:], (last.float() * 2).to(BF16)) and bool((w[0] == 0).all())
    # 64 rows whose logits are zero but for the last 64 words
    o = det.alloc_vocab_loss(64)
    work = det.alloc_vocab_loss_work(64, V, d, grad=True)
    grad = {"weight": torch.empty_like(w)}
    det.vocab_loss(last, w, t, o, work)
    det.vocab_loss_grad(last, w, t, o, grad, work, grad_rows=torch.ones(64, device="cuda"))
    ref = refs.Loss(last.cpu(), w[-64:].cpu(), torch.arange(64), grad_rows=torch.ones(64))
    logits = last.double() @ w[-64:].double().T
    lse = torch.logsumexp(torch.cat([logits, torch.full((64, 1), float(np.log(V - 64)), dtype=torch.float64, device="cuda")], 1), 1).cpu()
    within(o["lse"], lse, ref.lse_bound + V / 8192 * 2 * refs.U32 + 40 * refs.U32, "lse")
    g = torch.exp(logits.cpu() - lse[:, None]) - torch.eye(64, dtype=torch.float64)
    want = g.T @ last.double().cpu()
    err = (refs.u(BF16) * 1.01 + 1e-5) * (g.abs().T @ last.double().cpu().abs())
    within(grad["weight"][-64:], want, err + refs.u(BF16) * (want.abs() + err), "weight")
